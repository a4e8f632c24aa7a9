// One index for each row of scores: temperature, top-k, top-p and min-p, and a draw by
// the largest w_i / noise_i, which is a draw from w when the noise is exponential (the
// smallest of exponentials of rates w_i belongs to i with probability w_i / sum w), so
// no running sum over the row is needed to draw.
//
// Bound by memory when little is done for each entry: scores are read from memory once
// (a block's share of a row stays in shared memory as far as it fits, the rest comes
// again from L2) and noise only for entries that stay. A row belongs to a cluster of 1
// to 8 blocks. What top-k and top-p keep is a prefix of the order (score, larger first;
// index), so it is held as its last entry ("bound"). Three ways lead to it:
//   * no top-k, no top-p: every entry stays, and one pass after the maximum draws.
//   * small top-k: the k-th largest of the threads' own maxima is at most the k-th
//     largest score, so few entries lie at or above it; they are collected and ordered,
//     and all that follows works on k entries.
//   * else a histogram over (s_max - s) / T in equal steps finds the step in which the
//     prefix ends. Its entries are collected and ordered while the entries before it are
//     drawn from; where they are too many (rows of equal scores) the step is split again
//     by the bytes of the score and at last by those of the index.
// The inner loops work with w to about 1e-6 (one exp2); a candidate for the draw that comes
// within 4e-5 of the best so far is computed again in full. Sums that decide are
// integers, so that no result depends on the order of atomics: a step's w is its first
// value times (entries - sum of what each lacks to it, in steps of 2^-20).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "emr_act.h"
#include "emr_q8.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;
typedef unsigned long long u64;

constexpr int kMaxCluster = 8;
constexpr float kSpan = 24.f;    // the equal steps cover w in (e^-24, 1]; the last one takes the rest
constexpr float kNear = 4e-5f;   // of the draw's first computation
constexpr float kLackUnit = 1048576.f;

struct Args {
  const void* scores;
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
  int32_t room;                  // entries of a slice that shared memory holds
  int32_t vector, noise_vector;  // four entries at a time
  int32_t fix;                   // sums of w are kept in steps of 2^-fix
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
struct Mass {
  float sum, unused;
};

template <typename T>
struct Row {
  cg::cluster_group cluster;
  const Args& a;
  int tid, threads, lane, warp, warps, rank, blocks, phase;
  int64_t lo;       // first entry of this block's slice
  int count, held;  // its entries, and those in shared memory
  const T* global;  // the slice in memory
  T* data;          // and in shared memory
  const float* noise;
  uint32_t *counts, *lacks;
  u64 *sums, *list, *sorted;
  u64* scratch;     // [64]
  u64* slots;       // [2][kMaxCluster]
  int* list_size;
  float s_max, temperature, min_w, exp2_per;
  bool top_infinite;  // only the entries of +infinity count, as score 0
  // the draw
  Best best;
  float bar, mass;

  __device__ __forceinline__ float value(T v) const {
    const float s = float(v);
    return top_infinite ? (s == INFINITY ? 0.f : -INFINITY) : s;
  }
  // fn(score, entry of the slice) for every entry of this block, four at a time.
  template <typename Fn>
  __device__ __forceinline__ void each(Fn fn) const {
    each4([&](const float(&s)[4], int i, int have) {
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (j < have) fn(s[j], i + j);
    });
  }
  template <typename Fn>
  __device__ __forceinline__ void each4(Fn fn) const {
    for (int i = tid * 4; i < count; i += threads * 4) {
      const int have = count - i < 4 ? count - i : 4;
      float s[4];
      if (i < held || (a.vector && have == 4)) {  // held entries end at a multiple of 4 or with the slice
        Four<T> u;
        if (i < held) u.load(data + i);
        else u.load(global + i);
        const float4 f = u.floats();
        s[0] = f.x, s[1] = f.y, s[2] = f.z, s[3] = f.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++) s[j] = j < have ? float(global[i + j]) : -INFINITY;
      }
      if (top_infinite) {
#pragma unroll
        for (int j = 0; j < 4; j++) s[j] = s[j] == INFINITY ? 0.f : -INFINITY;
      }
      fn(s, i, have);
    }
  }
  __device__ __forceinline__ float weight(float s) const { return expf(__fdiv_rn(s - s_max, temperature)); }
  __device__ __forceinline__ float rough_weight(float s) const { return fast_exp2((s - s_max) * exp2_per); }
  __device__ __forceinline__ u64 fixed(float w) const { return __float2ull_rn(w * __int_as_float((127 + a.fix) << 23)); }
  __device__ __forceinline__ float step_at(float s, float per) const { return fminf((s_max - s) * per, float(a.bins - 1)); }

  __device__ void sync() {
    if (blocks > 1) cluster.sync();
    else __syncthreads();
  }
  template <typename V>
  __device__ __forceinline__ static V shfl_xor(V v, int o) {
    u64 u;
    memcpy(&u, &v, 8);
    u = __shfl_xor_sync(0xffffffffu, u, o);
    memcpy(&v, &u, 8);
    return v;
  }
  // Reduction over the row's threads, in an order of its own; every thread gets the result.
  template <typename V, typename Op>
  __device__ V reduce_block(V v, Op op) {
    static_assert(sizeof(V) == 8, "slots hold 8 bytes");
#pragma unroll
    for (int o = 16; o; o >>= 1) v = op(v, shfl_xor(v, o));
    __syncthreads();
    V* const part = reinterpret_cast<V*>(scratch);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    v = part[lane < warps ? lane : 0];
    for (int o = warps >> 1; o; o >>= 1) v = op(v, shfl_xor(v, o));  // warps is a power of two
    u64 u;
    memcpy(&u, &v, 8);
    u = __shfl_sync(0xffffffffu, u, 0);
    memcpy(&v, &u, 8);
    return v;
  }
  template <typename V, typename Op>
  __device__ V reduce(V v, Op op) {
    v = reduce_block(v, op);
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
    u64 part = lane < warps ? scratch[lane] : 0, sum = part;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 u = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += u;
    }
    *total = __shfl_sync(0xffffffffu, sum, 31);
    return __shfl_sync(0xffffffffu, sum - part, warp) + in - v;
  }
  // Largest of a value over the block.
  __device__ u64 block_max(u64 v) {
    return reduce_block(v, [](u64 x, u64 y) { return x > y ? x : y; });
  }

  __device__ __forceinline__ bool kept(uint32_t key, int64_t at, uint32_t bound_key, int64_t bound_at) const {
    return key > bound_key || (key == bound_key && key != 0 && at <= bound_at);
  }

  // ---- lists -----------------------------------------------------------------------------

  __device__ void list_clear() {
    if (tid == 0) *list_size = 0;
    sync();
  }
  // One entry to the list of the row's first block (dropped past its room, but counted).
  __device__ __forceinline__ void list_add(uint32_t key, int64_t at) {
    int* const size = blocks > 1 ? cluster.map_shared_rank(list_size, 0) : list_size;
    u64* const to = blocks > 1 ? cluster.map_shared_rank(list, 0) : list;
    const int place = atomicAdd(size, 1);
    if (place < a.cap) to[place] = (u64(key) << 32) | uint32_t(~uint32_t(at));
  }
  __device__ int list_end() {
    sync();
    const int got = blocks > 1 ? *cluster.map_shared_rank(list_size, 0) : *list_size;
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
#pragma unroll 8
        for (int i = 0; i < m; i++) place += list[i] > e;
        sorted[place] = e;
      }
    __syncthreads();
  }

  // ---- histograms ------------------------------------------------------------------------

  struct Found {
    int bin;
    int64_t size;  // entries of the step
    u64 before;    // entries, or w, before it
    u64 target;
  };
  // Of `bins` steps, summed over the row (value(b) their entries or w, size(b) their entries): the
  // last one with entries before which less than the target lies. by_mass with target 0: p
  // times the whole.
  template <typename Value, typename Size>
  __device__ Found locate(bool by_mass, int bins, u64 target, double p, u64 base, Value value, Size size) {
    const int per = (bins + threads - 1) / threads, b0 = tid * per;
    u64 mine = 0, total = 0;
    for (int b = b0; b < b0 + per && b < bins; b++) mine += value(b);
    u64 before = base + scan(mine, &total);
    Found f{-1, 0, 0, target};
    if (by_mass && target == 0) {
      const double t = ceil(double(total) * p);
      f.target = t < 1. ? 1 : u64(t);  // one entry stays at least
    }
    u64 pick = 0, pick_before = 0, pick_size = 0;  // pick: (bin + 1) of a candidate
    for (int b = b0; b < b0 + per && b < bins; b++) {
      const u64 c = size(b);
      if (c && before < f.target) pick = u64(b) + 1, pick_before = before, pick_size = c;
      before += value(b);
    }
    const u64 last = block_max(pick);  // every block finds the same
    __syncthreads();
    if (pick && pick == last) scratch[0] = pick_before, scratch[1] = pick_size;
    __syncthreads();
    f.bin = int(last) - 1;
    f.before = scratch[0];
    f.size = last ? int64_t(scratch[1]) : 0;
    sync();  // histograms are read before they are cleared
    return f;
  }
  __device__ __forceinline__ u64 over_blocks(const uint32_t* c, int b) const {
    u64 v = 0;
    for (int r = 0; r < blocks; r++) v += blocks > 1 ? cluster.map_shared_rank(c, r)[b] : c[b];
    return v;
  }
  // By steps given by bin(score, key, index), with w in full integers.
  template <typename In, typename Bin>
  __device__ Found find(bool by_mass, int bins, u64 target, In in, Bin bin, u64 base) {
    for (int i = tid; i < bins; i += threads) counts[i] = 0, sums[i] = 0;
    __syncthreads();
    each([&](float s, int i) {
      const uint32_t key = order_key(s);
      if (key && in(key, lo + i)) {
        const int at = bin(s, key, lo + i);
        atomicAdd(&counts[at], 1u);
        if (by_mass) atomicAdd(&sums[at], fixed(weight(s)));
      }
    });
    sync();
    return locate(by_mass, bins, target, 0., base,
                  [&](int b) {
                    if (!by_mass) return over_blocks(counts, b);
                    u64 v = 0;
                    for (int r = 0; r < blocks; r++) v += blocks > 1 ? cluster.map_shared_rank(sums, r)[b] : sums[b];
                    return v;
                  },
                  [&](int b) { return over_blocks(counts, b); });
  }
  // By equal steps of (s_max - s) / T.
  template <typename In>
  __device__ Found find_step(bool by_mass, u64 target, double p, float per, In in) {
    for (int i = tid; i < a.bins; i += threads) counts[i] = 0, lacks[i] = 0;
    __syncthreads();
    const float width = kSpan / float(a.bins - 1);
    const int last = a.bins - 1;
    float rest = 0.f;
    each([&](float s, int i) {
      if (!(s > -INFINITY) || !in(s, lo + i)) return;
      const float t = step_at(s, per);
      const int at = int(t);
      atomicAdd(&counts[at], 1u);
      if (by_mass) {
        if (at == last) {
          rest += rough_weight(s);
        } else {  // 1 - e^-x to x^4 / 24 < 3e-7
          const float x = (t - float(at)) * width;
          atomicAdd(&lacks[at], uint32_t(x * fmaf(x, fmaf(x, 1.f / 6.f, -0.5f), 1.f) * kLackUnit + 0.5f));
        }
      }
    });
    if (by_mass) rest = reduce(Mass{rest, 0.f}, [](Mass x, Mass y) { return Mass{x.sum + y.sum, 0.f}; }).sum;
    sync();
    return locate(by_mass, a.bins, target, p, 0,
                  [&](int b) {
                    const u64 c = over_blocks(counts, b);
                    if (!by_mass) return c;
                    if (b == last) return fixed(rest);
                    const float parts = float((c << 20) - over_blocks(lacks, b));
                    return __float2ull_rn(parts * expf(float(b) * -width) * __int_as_float((127 + a.fix - 20) << 23));
                  },
                  [&](int b) { return over_blocks(counts, b); });
  }

  // ---- selection -------------------------------------------------------------------------

  // Moves the bound (key, index) to the end of the prefix: `k` entries, or, by mass, the entries
  // before which less than p times the kept w lies. With by_mass the entries of the steps
  // before the last are drawn from on the way, and *drawn tells that only the list remains.
  __device__ void select(bool by_mass, int64_t k, double p, uint32_t& bound_key, int64_t& bound_at, bool* drawn) {
    const uint32_t bk = bound_key;
    const int64_t ba = bound_at;
    const float bs = bk ? key_score(bk) : -INFINITY;
    const float per = fminf(float(a.bins - 1) / (kSpan * temperature), 3e38f);
    Found f = find_step(by_mass, by_mass ? 0 : u64(k), p, per, [&](float s, int64_t at) { return s > bs || (s == bs && at <= ba); });
    const u64 target = f.target;
    const int step = f.bin;
    uint32_t prefix = 0;
    int shift = 32;  // key bits from `shift` up are fixed to prefix
    auto in = [&](uint32_t key, int64_t at) {
      return kept(key, at, bk, ba) && (shift == 32 || (key >> shift) == prefix) && int(step_at(key_score(key), per)) == step;
    };
    u64 before = f.before;
    int64_t size = f.size;
    while (size > a.cap && shift > 0) {
      const int next = shift - 8;
      // larger bytes first
      f = find(by_mass, 256, target, in, [&](float, uint32_t key, int64_t) { return 255 - int((key >> next) & 255u); }, before);
      prefix = (prefix << 8) | uint32_t(255 - f.bin);
      shift = next;
      before = f.before;
      size = f.size;
    }
    if (size <= a.cap) {
      const bool with_draw = by_mass && shift == 32;
      list_clear();
      if (with_draw) {
        *drawn = true;
        draw4([&](float s, int64_t at) {
          if (!(s > bs || (s == bs && at <= ba))) return false;
          const int b = int(step_at(s, per));
          if (b == step) list_add(order_key(s), at);
          return b < step;
        });
      } else {
        each([&](float s, int i) {
          const uint32_t key = order_key(s);
          if (key && in(key, lo + i)) list_add(key, lo + i);
        });
      }
      const int m = list_end();
      order(m);
      u64 e = 0;
      if (rank == 0) {
        if (!by_mass) {
          e = sorted[int64_t(target) - int64_t(before) - 1];
        } else {
          // the last entry before which less than the target lies
          u64 run = before, found = 0;
          for (int j0 = 0; j0 < m; j0 += threads) {
            const int j = j0 + tid;
            u64 all;
            const float s = j < m ? key_score(uint32_t(sorted[j] >> 32)) : 0.f;
            const u64 w = j < m ? fixed(weight(s)) : 0;
            const u64 ahead = run + scan(w, &all);
            if (j < m && ahead < target) {
              found = u64(j) + 1;
              if (with_draw) consider(s, int64_t(uint32_t(~uint32_t(sorted[j]))), noise[uint32_t(~uint32_t(sorted[j]))]);
            }
            run += all;
          }
          found = block_max(found);
          e = sorted[found - 1];
        }
      }
      if (with_draw) return;  // nothing more asks for the bound
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
      want = w == 0 ? size : int64_t((target - before + w - 1) / w);
      want = want < 1 ? 1 : want > size ? size : want;
    }
    uint32_t ahead = 0;
    u64 passed = 0;
    for (int next = 24; next >= 0; next -= 8) {
      const int above = next + 8;
      const uint32_t fixed_bits = ahead;
      f = find(false, 256, u64(want),
               [&](uint32_t x, int64_t at) { return x == key && at <= (x == bk ? ba : INT64_MAX) && (above == 32 || (uint32_t(at) >> above) == fixed_bits); },
               [&](float, uint32_t, int64_t at) { return int((uint32_t(at) >> next) & 255u); }, passed);
      ahead = (ahead << 8) | uint32_t(f.bin);
      passed = f.before;
    }
    bound_key = key;
    bound_at = int64_t(ahead);
  }

  // A score that is at most the k-th largest of the row (its key), from the threads' own largest.
  __device__ uint32_t floor_key(uint32_t own, int k) {
    uint32_t prefix = 0, before = 0;
#pragma unroll
    for (int shift = 24; shift >= 16; shift -= 8) {
      for (int i = tid; i < 256; i += threads) counts[i] = 0;
      __syncthreads();
      if (own && (shift == 24 || (own >> 24) == prefix)) atomicAdd(&counts[255 - ((own >> shift) & 255u)], 1u);
      __syncthreads();
      u64 all;
      const u64 c = tid < 256 ? counts[tid] : 0, ahead = before + scan(c, &all);
      const u64 pick = block_max(tid < 256 && c && ahead < u64(k) ? (u64(tid) + 1) << 32 | ahead : 0);
      if (before + all < u64(k)) return 1;  // fewer threads than k have an entry
      prefix = prefix << 8 | (255 - uint32_t((pick >> 32) - 1));
      before = uint32_t(pick);
      __syncthreads();
    }
    return prefix << 16;
  }

  // ---- the draw --------------------------------------------------------------------------

  __device__ __forceinline__ void consider(float s, int64_t at, float e) {
    const float w = rough_weight(s);
    if (w >= min_w) mass += w;
    if (w * fast_rcp(e) > bar) {
      const float exact = weight(s);
      if (exact >= min_w) {
        best = better(best, Best{exact > 0.f ? __fdiv_rn(exact, e) : 0.f, int32_t(at)});
        bar = best.key * (1.f - kNear);
      }
    }
  }
  // Draws from the entries for which in(score, index) holds.
  template <typename In>
  __device__ __forceinline__ void draw4(In in) {
    each4([&](const float(&s)[4], int i, int have) {
      bool stay[4];
      bool any = false;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        stay[j] = j < have && s[j] > -INFINITY && in(s[j], lo + i + j);
        any |= stay[j];
      }
      if (!any) return;
      float e[4];
      if (a.noise_vector && have == 4) {
        const float4 f = __ldcs(reinterpret_cast<const float4*>(noise + lo + i));
        e[0] = f.x, e[1] = f.y, e[2] = f.z, e[3] = f.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++) e[j] = stay[j] ? noise[lo + i + j] : 1.f;
      }
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (stay[j]) consider(s[j], lo + i + j, e[j]);
    });
  }
  __device__ void finish(int32_t* index, float* logp) {
    const Best top = reduce(best, [](Best x, Best y) { return better(x, y); });
    const float sum = reduce(Mass{mass, 0.f}, [](Mass x, Mass y) { return Mass{x.sum + y.sum, 0.f}; }).sum;
    if (top.at < 0) {  // no positive noise among what stays
      if (rank == 0 && tid == 0) {
        *index = -1;
        if (logp) *logp = -INFINITY;
      }
    } else if (top.at >= lo && top.at < lo + count && tid == 0) {
      *index = top.at;
      if (logp) *logp = __fdiv_rn(value(global[top.at - lo]) - s_max, temperature) - logf(sum);
    }
  }
  // The first k of the list (m entries) hold all that stays: top-p and the draw on them, by the
  // row's first block.
  __device__ void finish_list(int k, int m, float p, int32_t* index, float* logp) {
    order(m);
    if (rank != 0) return;
    const int have = k < m ? k : m;
    u64 before = 0, total = 0, target = ~u64(0);
    const float s = tid < have ? key_score(uint32_t(sorted[tid] >> 32)) : 0.f;
    const int64_t at = tid < have ? int64_t(uint32_t(~uint32_t(sorted[tid]))) : 0;
    if (p < 1.f) {
      before = scan(tid < have ? fixed(weight(s)) : 0, &total);
      const double t = ceil(double(total) * double(p));
      target = t < 1. ? 1 : u64(t);
    }
    if (tid < have && before < target) consider(s, at, noise[at]);
    const Best top = reduce_block(best, [](Best x, Best y) { return better(x, y); });
    const float sum = reduce_block(Mass{mass, 0.f}, [](Mass x, Mass y) { return Mass{x.sum + y.sum, 0.f}; }).sum;
    if (top.at < 0) {
      if (tid == 0) {
        *index = -1;
        if (logp) *logp = -INFINITY;
      }
    } else if (tid < have && at == top.at) {
      *index = top.at;
      if (logp) *logp = __fdiv_rn(s - s_max, temperature) - logf(sum);
    }
  }
};

// kFree: neither top-k nor top-p for any row.
template <typename T, int kThreads, bool kFree>
__global__ void __launch_bounds__(kThreads, 2048 / kThreads > 4 ? 4 : kThreads == 512 ? 2 : 1) sample_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ u64 scratch[64], slots[2 * kMaxCluster];
  __shared__ int list_size;
  Row<T> r{cg::this_cluster(), a};
  r.tid = threadIdx.x, r.threads = kThreads, r.lane = r.tid & 31, r.warp = r.tid >> 5, r.warps = kThreads / 32;
  r.rank = int(r.cluster.block_rank()), r.blocks = int(r.cluster.num_blocks()), r.phase = 0;
  r.scratch = scratch, r.slots = slots, r.list_size = &list_size;
  r.sums = reinterpret_cast<u64*>(smem);  // the first 256 steps; shares its memory with lacks
  r.lacks = reinterpret_cast<uint32_t*>(smem);
  r.counts = r.lacks + a.bins;
  r.sorted = r.sums;  // the histogram is done with when entries are ordered
  r.list = reinterpret_cast<u64*>(r.counts + a.bins);
  r.data = reinterpret_cast<T*>(r.list + a.cap);
  const int64_t row = blockIdx.x / unsigned(r.blocks);
  r.lo = r.rank * a.slice;
  r.count = int(a.n - r.lo < 0 ? 0 : a.n - r.lo < a.slice ? a.n - r.lo : a.slice);
  r.held = 0;
  r.global = static_cast<const T*>(a.scores) + row * a.row_stride + r.lo;
  r.noise = a.noise + row * a.noise_stride;
  r.top_infinite = false;
  r.best = Best{-1.f, -1}, r.bar = -1.f, r.mass = 0.f;
  int32_t* index = a.index + row;
  float* logp = a.logp ? a.logp + row : nullptr;

  // scores once from memory: the thread's largest, and into shared memory
  float top = -INFINITY;
#pragma unroll 4
  for (int i = r.tid * 4; i < r.count; i += kThreads * 4) {
    Four<T> u;
    if (a.vector && i + 4 <= r.count) {
      u.load(r.global + i);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) u.set(j, i + j < r.count ? r.global[i + j] : T(-INFINITY));
    }
    if (i < a.room) u.store(r.data + i);
    const float4 f = u.floats();
    top = fmaxf(fmaxf(top, fmaxf(f.x, f.y)), fmaxf(f.z, f.w));  // NaN is passed over
  }
  r.held = r.count < a.room ? r.count : a.room;
  const uint32_t own = order_key(top);
  const u64 top_key = r.reduce(u64(own), [](u64 x, u64 y) { return x > y ? x : y; });
  if (top_key == 0) {  // nothing left
    if (r.rank == 0 && r.tid == 0) {
      *index = -1;
      if (logp) *logp = -INFINITY;
    }
    return;
  }
  r.s_max = key_score(uint32_t(top_key));
  if (r.s_max == INFINITY) r.top_infinite = true, r.s_max = 0.f;
  r.temperature = a.temperature ? a.temperature[row] : a.temperature_all;
  r.min_w = fminf(a.min_p ? a.min_p[row] : a.min_p_all, 1.f);
  r.exp2_per = fminf(kLog2E / r.temperature, 3e38f);
  const int64_t k = kFree ? 0 : a.top_k ? a.top_k[row] : a.top_k_all;
  const float p = kFree ? 1.f : a.top_p ? a.top_p[row] : a.top_p_all;
  __syncthreads();  // the scores are in shared memory

  if (!(r.temperature > 0.f)) {  // the largest score
    int64_t at = INT64_MAX;
    r.each([&](float s, int i) {
      if (s == r.s_max && r.lo + i < at) at = r.lo + i;
    });
    at = r.reduce(at, [](int64_t x, int64_t y) { return x < y ? x : y; });
    if (r.rank == 0 && r.tid == 0) {
      *index = int32_t(at);
      if (logp) *logp = 0.f;
    }
    r.sync();
    return;
  }
  if constexpr (kFree) {
    r.draw4([](float, int64_t) { return true; });
    r.finish(index, logp);
  } else {
    uint32_t bound_key = 0;
    int64_t bound_at = INT64_MAX;
    bool done = false;
    if (k > 0 && k < a.n) {
      if (k <= kThreads / 4) {
        // the k-th largest of one block's threads bounds the row's from below: the best of the blocks'
        const u64 least = r.reduce(u64(r.floor_key(r.top_infinite ? (top == INFINITY ? order_key(0.f) : 0) : own, int(k))),
                                   [](u64 x, u64 y) { return x > y ? x : y; });
        const float low = least > 1 ? key_score(uint32_t(least)) : -INFINITY;
        r.list_clear();
        r.each4([&](const float(&s)[4], int i, int have) {
          if (!(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) >= low)) return;
#pragma unroll
          for (int j = 0; j < 4; j++)
            if (j < have && s[j] >= low && s[j] > -INFINITY) r.list_add(order_key(s[j]), r.lo + i + j);
        });
        const int m = r.list_end();
        if (m <= a.cap) r.finish_list(int(k), m, p, index, logp), done = true;
      }
      if (!done) {
        // a score is masked or counted: where fewer than k are left all of them stay
        u64 valid = 0;
        r.each([&](float s, int) { valid += s > -INFINITY; });
        valid = r.reduce(valid, [](u64 x, u64 y) { return x + y; });
        if (u64(k) < valid) r.select(false, k, 0., bound_key, bound_at, nullptr);
      }
    }
    if (!done) {
      bool drawn = false;
      if (p < 1.f) r.select(true, 0, double(p), bound_key, bound_at, &drawn);
      if (!drawn) {
        const float bs = bound_key ? key_score(bound_key) : -INFINITY;
        r.draw4([&](float s, int64_t at) { return s > bs || (s == bs && at <= bound_at); });
      }
      r.finish(index, logp);
    }
  }
  r.sync();  // no block ends while another may still read its memory
}

template <typename T, int kThreads, bool kFree>
emr_status launch(const Args& a, int rows, int cluster, size_t smem, int dev, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(sample_kernel<T, kThreads, kFree>, kMostSmem, dev, done)) return EMR_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(rows) * unsigned(cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = unsigned(cluster);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, kThreads, kFree>, a) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

template <typename T>
emr_status plan(Args a, int rows, bool free, int dev, int sms, cudaStream_t st) {
  // Blocks of a row: as many as find an SM each while a slice has 2048 entries.
  int cluster = 1;
  while (cluster < kMaxCluster && int64_t(rows) * (cluster + 1) <= sms && a.n / (cluster + 1) >= 2048) cluster++;
  a.slice = ((a.n + cluster - 1) / cluster + 15) / 16 * 16;
  const bool wide = a.slice > 8192, crowd = int64_t(rows) * cluster > sms;
  // Shared memory of a block: all of an SM's, half where two blocks of 512 threads share one,
  // and what a short slice needs.
  a.bins = free ? 0 : !wide ? 512 : crowd ? 2048 : 4096;
  a.cap = free ? 0 : !wide ? 512 : crowd ? 1024 : 2048;
  size_t smem = size_t(a.bins) * 8 + size_t(a.cap) * 8;
  const size_t most = wide && !crowd ? kMostSmem : 112 * 1024;
  const size_t want = size_t(a.slice) * sizeof(T), room = most > smem ? most - smem : 0;
  a.room = int32_t((want < room ? want : room) / sizeof(T) / 4 * 4);
  smem += size_t(a.room) * sizeof(T);
  const int threads = !wide ? 256 : crowd ? 512 : 1024;
  if (free)
    return threads == 256 ? launch<T, 256, true>(a, rows, cluster, smem, dev, st)
           : threads == 512 ? launch<T, 512, true>(a, rows, cluster, smem, dev, st) : launch<T, 1024, true>(a, rows, cluster, smem, dev, st);
  return threads == 256 ? launch<T, 256, false>(a, rows, cluster, smem, dev, st)
         : threads == 512 ? launch<T, 512, false>(a, rows, cluster, smem, dev, st) : launch<T, 1024, false>(a, rows, cluster, smem, dev, st);
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
      reinterpret_cast<uintptr_t>(index) % 4 || reinterpret_cast<uintptr_t>(logp) % 4 || reinterpret_cast<uintptr_t>(temperature) % 4 ||
      reinterpret_cast<uintptr_t>(top_k) % 4 || reinterpret_cast<uintptr_t>(top_p) % 4 || reinterpret_cast<uintptr_t>(min_p) % 4)
    return EMR_ERR_ARG;
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  Args a{};
  a.scores = scores, a.n = n, a.row_stride = row_stride, a.noise = noise, a.noise_stride = noise_stride;
  a.temperature = temperature, a.top_k = top_k, a.top_p = top_p, a.min_p = min_p;
  a.temperature_all = temperature_all, a.top_k_all = top_k_all, a.top_p_all = top_p_all, a.min_p_all = min_p_all;
  a.index = index, a.logp = logp;
  int bits = 0;
  while ((int64_t(1) << bits) < n) bits++;
  a.fix = bits <= 18 ? 44 : 62 - bits;
  a.vector = reinterpret_cast<uintptr_t>(scores) % (4 * size) == 0 && (rows == 1 || row_stride % 4 == 0);
  a.noise_vector = reinterpret_cast<uintptr_t>(noise) % 16 == 0 && (rows == 1 || noise_stride % 4 == 0);
  const bool free = !top_k && !top_p && (top_k_all <= 0 || top_k_all >= n) && !(top_p_all < 1.f);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == EMR_F32) return plan<float>(a, rows, free, dev, sms, st);
  if (dtype == EMR_BF16) return plan<__nv_bfloat16>(a, rows, free, dev, sms, st);
  return plan<__half>(a, rows, free, dev, sms, st);
}
