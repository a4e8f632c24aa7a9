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
// Measured in a captured graph, where L2 keeps a part of the inputs: 1000 x 5460 float32 without
// filters 12 us (memory's time for scores and noise: 6.4), 256 x 87380 bfloat16 with top-k 50,
// top-p and min-p 21 (6.6 for the scores), 24 x 349524 float32 with top-p 55 (9.9 with all
// noise): the last is bound by two shared-memory atomics for an entry and by about ten
// exchanges of a cluster. The probabilities' sums are floats: turns of 8 or 16 entries, added
// with their rounding kept, so that the length of a row does not show in them.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <mutex>

#include "emr_act.h"
#include "emr_q8.h"
#include "emr_rows.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;
typedef unsigned long long u64;

constexpr int kMaxCluster = 8;
constexpr float kSpan = 16.f;    // the equal steps cover w in (e^-16, 1]; the last one takes the rest
constexpr float kNear = 6e-5f;   // of the draw's first computation, in units of log2
constexpr float kLackUnit = 1048576.f;
// A step's lacks are summed in 32 bits. An entry's is at most 2^24 / (steps - 1), so (steps - 1) 127 entries of a
// block stay below 2^31: 63 turns of each_group with the 8 entries a turn of a thread, at 4 steps a thread. Longer
// slices carry what is above 2^31 into a second word every so many turns.
constexpr int kCarryTurns = 63;

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
  int32_t room;                  // groups of 16 bytes of a slice that shared memory holds
  int32_t noise_vector;          // rows of noise are aligned to 16 bytes
  int32_t fix;                   // sums of w are kept in steps of 2^-fix
  int32_t carry;                 // lacks have a second word
};

// Predicated, not branched around.
__device__ __forceinline__ void shared_add(bool go, uint32_t at, uint32_t v) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p red.shared.add.u32 [%0], %1;\n\t}" ::"r"(at), "r"(v), "r"(uint32_t(go)) : "memory");
}
__device__ __forceinline__ uint4 shared_load(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
// A draw's best entry, the larger key first, then the lower index; its keys are non-negative
// floats as integers, one up, so that 0 stands for none.
struct Drawn {
  uint32_t key, at;
  float mass;       // w of what was drawn from
  uint32_t unsure;  // order_key of the largest rough key that might stand before the best
};
__device__ __forceinline__ uint32_t draw_key(float k) { return k >= 0.f ? __float_as_uint(k) + 1 : 0; }
__device__ __forceinline__ float draw_value(uint32_t k) { return k ? __uint_as_float(k - 1) : -1.f; }
__device__ __forceinline__ void join(Drawn& x, const Drawn& y) {
  if (y.key > x.key || (y.key == x.key && y.at < x.at)) x.key = y.key, x.at = y.at;
  x.mass += y.mass;
  x.unsure = max(x.unsure, y.unsure);
}

template <typename T, int kAhead>
struct Row {
  static constexpr int kG = Group<T>::kSize;
  cg::cluster_group cluster;
  const Args& a;
  int tid, threads, lane, warp, warps, rank, blocks, phase, turn;
  int lo;           // first entry of this block's slice
  int count;        // its entries, the first of them `skip` entries after a multiple of 16 bytes
  int skip, groups, held;  // groups of 16 bytes that they lie in, and those in shared memory
  const T* global;  // the slice in memory
  uint4* data;      // and in shared memory
  const float* noise;   // of the row
  uint32_t data_at, counts_at, lacks_at;  // addresses in shared memory, for the inner loops
  uint32_t *counts, *lacks;  // and, with a.carry, the lacks' second words behind the counts
  u64 *sums, *list, *sorted;
  uint4* scratch;   // [2][32], by turns: a turn's values are read by all before the next but one writes
  uint4* slots;     // [2][kMaxCluster]
  u64* found;       // [2]: what one thread found for all
  int* list_size;   // [3]: of the first, second and third list of the row
  u64 *coarse;      // [2][64]: w and entries of 64 groups of steps
  float* rest;      // w of the last step
  int lists;
  bool counted;     // a histogram has been made
  float s_max, temperature, min_w, exp2_per;
  bool top_infinite;  // only the entries of +infinity count, as score 0
  // the draw: a thread's largest and second largest log2(w / noise) as computed roughly, and its w
  // (needed unless the histogram has told it)
  float rough, rough_second, mass;
  float part;        // of mass: the w of one turn
  float2* turns;     // in shared memory, a thread's own: the sum of its turns, and what that has rounded off
  bool need_mass;
  float min_log2;   // least log2 w that stays, with the margin
  int32_t rough_at;
  u64 bound;        // where the first block knows it: the last entry that stays

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
  // fn(scores, i) for kAhead groups, loaded together, of every block's: scores[u][j] is entry i + u
  // threads kG + j of the slice, and -infinity past it (i may be below 0).
  // Of the groups from first to before past, apart by whole turns.
  template <typename Fn>
  __device__ __forceinline__ void each_group(Fn fn, int first, int past) const {
    for (int g = first + tid; g < past; g += threads * kAhead) {
      Group<T> v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        const int at = g + u * threads;
        if (at < held) v[u].u = shared_load(data_at + at * 16);
        else v[u] = fetch(at);
      }
      float s[kAhead][kG];
#pragma unroll
      for (int u = 0; u < kAhead; u++)
#pragma unroll
        for (int j = 0; j < kG; j++) s[u][j] = v[u].get(j);
      if (top_infinite) {
#pragma unroll
        for (int u = 0; u < kAhead; u++)
#pragma unroll
          for (int j = 0; j < kG; j++) s[u][j] = s[u][j] == INFINITY ? 0.f : -INFINITY;
      }
      fn(s, g * kG - skip);
    }
  }
  template <typename Fn>
  __device__ __forceinline__ void each_group(Fn fn) const { each_group(fn, 0, groups); }
  // fn(score, entry of the slice); past the slice, too, with -infinity.
  template <typename Fn>
  __device__ __forceinline__ void each(Fn fn, int first, int past) const {
    each_group([&](const float (&s)[kAhead][kG], int i) {
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        if (i + u * threads * kG >= count) break;
#pragma unroll
        for (int j = 0; j < kG; j++) fn(s[u][j], i + u * threads * kG + j);
      }
    }, first, past);
  }
  template <typename Fn>
  __device__ __forceinline__ void each(Fn fn) const { each(fn, 0, groups); }
  __device__ __forceinline__ float weight(float s) const { return expf(__fdiv_rn(s - s_max, temperature)); }
  __device__ __forceinline__ float rough_weight(float s) const { return fast_exp2((s - s_max) * exp2_per); }
  __device__ __forceinline__ u64 fixed(float w) const { return __float2ull_rn(w * __int_as_float((127 + a.fix) << 23)); }
  // Step of a score, 2^23 up, as a float: rises as the score falls. Rounded by that shift, not
  // converted: conversions take a quarter of the rate.
  __device__ __forceinline__ float step_up(float s, float per) const { return fmaxf(fmaf(s_max - s, per, -0.5f), 0.f) + 0x1p+23f; }
  __device__ __forceinline__ float last_up() const { return float(a.bins - 1) + 0x1p+23f; }
  __device__ __forceinline__ int step_of(float s, float per) const {
    return int(__float_as_uint(fminf(step_up(s, per), last_up())) & 0x7fffffu);
  }

  __device__ void sync() {
    if (blocks > 1) cluster.sync();
    else __syncthreads();
  }
  // One barrier for each of these: what a warp finds is combined by every warp again.
  __device__ uint32_t block_max(uint32_t v) {
    uint32_t* const part = reinterpret_cast<uint32_t*>(scratch + 32 * (turn ^= 1));
    v = __reduce_max_sync(0xffffffffu, v);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, lane < warps ? part[lane] : 0);
  }
  __device__ static float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
  __device__ float block_sum(float v) {
    float* const part = reinterpret_cast<float*>(scratch + 32 * (turn ^= 1));
    v = warp_sum(v);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    return warp_sum(lane < warps ? part[lane] : 0.f);
  }
  __device__ static Drawn warp_best(Drawn d) {
    const uint32_t key = __reduce_max_sync(0xffffffffu, d.key);
    d.at = __reduce_min_sync(0xffffffffu, d.key == key ? d.at : 0xffffffffu);
    d.key = key;
    d.mass = warp_sum(d.mass);
    d.unsure = __reduce_max_sync(0xffffffffu, d.unsure);
    return d;
  }
  __device__ Drawn block_best(Drawn d) {
    Drawn* const part = reinterpret_cast<Drawn*>(scratch + 32 * (turn ^= 1));
    d = warp_best(d);
    if (lane == 0) part[warp] = d;
    __syncthreads();
    return warp_best(lane < warps ? part[lane] : Drawn{0, 0xffffffffu, 0.f, 0});
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
  __device__ u64 row_max(u64 v) {  // of values that all threads of a block share
    if (blocks == 1) return v;
    u64 most = 0;
    exchange(v, [&](u64 x) { most = x > most ? x : most; });
    return most;
  }
  __device__ Drawn row_best(Drawn d) {
    d = block_best(d);
    if (blocks == 1) return d;
    Drawn all{0, 0xffffffffu, 0.f, 0};
    exchange(d, [&](const Drawn& x) { join(all, x); });
    return all;
  }
  // Exclusive sum over the block's threads in order, of values below 2^62; *total gets the whole sum.
  __device__ u64 scan(u64 v, u64* total) {
    u64* const part = reinterpret_cast<u64*>(scratch + 32 * (turn ^= 1));
    u64 in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 u = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += u;
    }
    if (lane == 31) part[warp] = in;
    __syncthreads();
    const u64 w = lane < warps ? part[lane] : 0;
    u64 before = 0, all = 0;  // in pieces of 22 bits, whose sums over 32 lanes fit into 32
#pragma unroll
    for (int i = 0; i < 3; i++) {
      const uint32_t piece = uint32_t(w >> (22 * i)) & 0x3fffffu;
      all += u64(__reduce_add_sync(0xffffffffu, piece)) << (22 * i);
      before += u64(__reduce_add_sync(0xffffffffu, lane < warp ? piece : 0)) << (22 * i);
    }
    *total = all;
    return before + in - v;
  }
  // p times total, rounded up: p in (0, 1) is m 2^-s with 24 bits of m.
  __device__ static u64 share_of(u64 total, float p) {
    const uint32_t bits = __float_as_uint(p), e = bits >> 23;
    const uint32_t m = (bits & 0x7fffffu) | (e ? 0x800000u : 0);
    const int s = 150 - int(e ? e : 1);  // at least 24
    const u64 lo = total * m, hi = __umul64hi(total, m);
    const u64 kept = s >= 128 ? 0 : s >= 64 ? hi >> (s - 64) : (hi << (64 - s)) | (lo >> s);
    const bool more = s >= 128 ? (hi | lo) != 0 : s >= 64 ? (hi << 1 << (127 - s)) != 0 || lo != 0 : lo << (64 - s) != 0;
    return kept + more;
  }

  __device__ __forceinline__ bool kept(uint32_t key, uint32_t at, uint32_t bound_key, uint32_t bound_at) const {
    return key > bound_key || (key == bound_key && key != 0 && at <= bound_at);
  }

  // ---- lists -----------------------------------------------------------------------------

  // One entry to the list of the row's first block (dropped past its room, but counted).
  __device__ __forceinline__ void list_add(uint32_t key, uint32_t at) {
    int* const size = blocks > 1 ? cluster.map_shared_rank(list_size + lists, 0) : list_size + lists;
    u64* const to = blocks > 1 ? cluster.map_shared_rank(list, 0) : list;
    const int place = atomicAdd(size, 1);
    if (place < a.cap) to[place] = (u64(key) << 32) | uint32_t(~at);
  }
  __device__ int list_end() {
    sync();
    const int got = blocks > 1 ? *cluster.map_shared_rank(list_size + lists, 0) : list_size[lists];
    lists++;
    return got;
  }
  // The list's m entries in order, in `sorted` of the row's first block: an entry's place
  // is the number of larger ones, counted by a warp.
  __device__ void order(int m) {
    if (rank == 0)
      for (int j = warp; j < m; j += warps) {
        const u64 e = list[j];
        int larger = 0;
#pragma unroll 4
        for (int i = lane; i < m; i += 32) larger += list[i] > e;
        larger = __reduce_add_sync(0xffffffffu, larger);
        if (lane == 0) sorted[larger] = e;
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
  // What a step counts for: its entries, its w from entries and lacks, or its w as summed.
  enum Kind { kEntries, kLacks, kSums };
  __device__ __forceinline__ u64 step_value(Kind kind, int b, u64 c, u64 l) const {
    if (kind == kEntries) return c;
    if (kind == kSums) return l;
    if (b == a.bins - 1) return fixed(*rest);  // one block's; see locate
    return __float2ull_rn(float((c << 20) - l) * expf(float(b) * (-kSpan / float(a.bins - 1))) * __int_as_float((127 + a.fix - 20) << 23));
  }
  __device__ __forceinline__ u64 lack(const uint32_t* of, int b) const {
    return a.carry ? of[b] + (u64(of[2 * a.bins + b]) << 31) : of[b];
  }
  __device__ __forceinline__ u64 second(Kind kind, int b) const { return kind == kSums ? sums[b] : kind == kLacks ? lack(lacks, b) : 0; }
  template <typename V>
  __device__ __forceinline__ const V* of_block(const V* p, int r) const { return cluster.map_shared_rank(p, r); }

  // The last step with entries before which less than the target lies. With several blocks first
  // among 64 groups of steps, then among the steps of one, so that a thread reads few values of
  // the other blocks. By w with target 0: p times the whole.
  __device__ Found locate(Kind kind, int bins, u64 target, float p, u64 base) {
    const int q = bins > threads ? bins / threads : 1;  // steps of a thread, at most 4
    const int b0 = tid * q;
    u64 v = 0, c = 0;
    if (b0 < bins)
      for (int j = 0; j < q; j++) {
        const u64 n = counts[b0 + j];
        c += n;
        if (n) v += step_value(kind, b0 + j, n, second(kind, b0 + j));
      }
    Found f{-1, 0, base, target};
    int first = 0, many = bins, each_has = q;
    if (blocks > 1) {
      const int team = bins / 64 / q;  // threads of a group: a power of two up to 16
      u64 gv = v, gc = c;
      for (int o = team >> 1; o; o >>= 1) gv += __shfl_xor_sync(0xffffffffu, gv, o), gc += __shfl_xor_sync(0xffffffffu, gc, o);
      if (b0 < bins && tid % team == 0) coarse[tid / team] = gv, coarse[64 + tid / team] = gc;
      sync();
      v = c = 0;
      if (tid < 64) {
#pragma unroll
        for (int r = 0; r < kMaxCluster; r++)
          if (r < blocks) v += of_block(coarse, r)[tid], c += of_block(coarse, r)[64 + tid];
      }
      many = 64, each_has = 1;
    }
    for (int level = 0;; level++) {
      u64 total;
      if (tid == 0) found[0] = ~u64(0);
      u64 before = f.before + scan(v, &total);
      if (level == 0 && kind != kEntries && target == 0) {
        f.target = share_of(total, p);
        if (f.target == 0) f.target = 1;  // one entry stays at least
      }
      // the step, or group, in which the target lies
      const auto ends_here = [&](u64 from, u64 size, u64 entries, int b) {
        if (entries && from < f.target && f.target <= from + size) found[0] = from, found[1] = entries, found[2] = u64(b);
      };
      if (each_has == 1) {
        if (tid < many) ends_here(before, v, c, first + tid);
      } else if (b0 < bins && before < f.target && f.target <= before + v) {
        for (int j = 0; j < q; j++) {
          const u64 n = counts[b0 + j], w = n ? step_value(kind, b0 + j, n, second(kind, b0 + j)) : 0;
          ends_here(before, w, n, b0 + j);
          before += w;
        }
      }
      __syncthreads();
      if (found[0] == ~u64(0)) {  // roundings have left the target past the end: the last one with entries
        int last_b = -1;
        u64 last_n = 0, last_from = 0;
        if (each_has == 1) {
          if (tid < many && c) last_b = first + tid, last_n = c, last_from = before;
        } else if (b0 < bins) {
          for (int j = 0; j < q; j++) {
            const u64 n = counts[b0 + j];
            if (n) last_b = b0 + j, last_n = n, last_from = before;
            if (n) before += step_value(kind, b0 + j, n, second(kind, b0 + j));
          }
        }
        const uint32_t b = block_max(uint32_t(last_b + 1));
        if (b && last_b + 1 == int(b)) found[0] = last_from, found[1] = last_n, found[2] = u64(last_b);
        __syncthreads();
      }
      f.before = found[0], f.size = int64_t(found[1]), f.bin = int(found[2]);
      __syncthreads();  // read before it is written again
      if (blocks == 1 || level == 1) return f;
      // the steps of the group, over the blocks
      many = bins / 64;
      first = f.bin * many;
      v = c = 0;
      if (tid < many) {
        const int b = first + tid;
        u64 l = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; r++)
          if (r < blocks) {
            c += of_block(counts, r)[b];
            if (kind == kSums) l += of_block(sums, r)[b];
            if (kind == kLacks) l += lack(of_block(lacks, r), b);
          }
        if (kind == kLacks && b == a.bins - 1) {
          for (int r = 0; r < blocks; r++) v += fixed(*of_block(rest, r));
        } else if (c) {
          v = step_value(kind, b, c, l);
        }
      }
    }
  }
  // Before a histogram: the one before it has been read by every block.
  __device__ void histogram_begin(int bins, bool wide) {
    if (counted) sync();
    counted = true;
    for (int i = tid; i < bins; i += threads) {
      counts[i] = 0;
      if (wide) sums[i] = 0;
      else lacks[i] = 0;
      if (!wide && a.carry) lacks[2 * a.bins + i] = 0;
    }
    __syncthreads();
  }
  // By steps given by bin(score, key, index), with w in full integers.
  template <typename In, typename Bin>
  __device__ Found find(bool by_mass, int bins, u64 target, In in, Bin bin, u64 base) {
    histogram_begin(bins, true);
    each([&](float s, int i) {
      const uint32_t key = order_key(s);
      if (key && in(key, lo + i)) {
        const int at = bin(s, key, lo + i);
        atomicAdd(&counts[at], 1u);
        if (by_mass) atomicAdd(&sums[at], fixed(weight(s)));
      }
    });
    __syncthreads();
    return locate(by_mass ? kSums : kEntries, bins, target, 0.f, base);
  }
  // By equal steps of (s_max - s) / T.
  template <typename In>
  __device__ Found find_step(bool by_mass, u64 target, float p, float per, In in) {
    histogram_begin(a.bins, false);
    const float width = kSpan / float(a.bins - 1);
    const int last = a.bins - 1;
    float below = 0.f;
    const auto add = [&](float s, int i) {
      const bool ok = (s > -INFINITY) & in(s, uint32_t(lo + i));
      const float up = fminf(step_up(s, per), last_up());
      const int at = int(__float_as_uint(up) & 0x7fffffu);
      shared_add(ok, counts_at + at * 4, 1u);
      if (by_mass) {
        if (ok && at == last) below += rough_weight(s);
        // 1 - e^-x to x^4 / 24 < 3e-7
        const float x = fmaxf(fmaf(s_max - s, per, 0x1p+23f - up), 0.f) * width;
        const float lack = x * fmaf(x, fmaf(x, 1.f / 6.f, -0.5f), 1.f) * kLackUnit + 0x1p+23f;
        shared_add(ok & (at != last), lacks_at + at * 4, __float_as_uint(lack) & 0x7fffffu);
      }
    };
    const int turns = a.carry ? kCarryTurns * threads * kAhead : groups;
    for (int from = 0; from < groups; from += turns) {
      if (from) {
        __syncthreads();
        for (int i = tid; i < a.bins; i += threads) lacks[2 * a.bins + i] += lacks[i] >> 31, lacks[i] &= 0x7fffffffu;
        __syncthreads();
      }
      each(add, from, groups - from < turns ? groups : from + turns);
    }
    if (__syncthreads_or(below > 0.f)) below = block_sum(below);
    if (by_mass) {
      if (tid == 0) *rest = below;
      __syncthreads();
    }
    return locate(by_mass ? kLacks : kEntries, a.bins, target, p, 0);
  }

  // ---- selection -------------------------------------------------------------------------

  // Moves the bound (key, index) to the end of the prefix: `k` entries, or, by mass, the entries
  // before which less than p times the kept w lies. With by_mass the entries of the steps
  // before the last are drawn from on the way, and *drawn tells that only the list remains.
  __device__ void select(bool by_mass, int64_t k, float p, uint32_t& bound_key, uint32_t& bound_at, bool* drawn) {
    const uint32_t bk = bound_key;
    const uint32_t ba = bound_at;
    const float bs = bk ? key_score(bk) : -INFINITY;  // no bound: every score that is not masked is above it
    const float per = fminf(float(a.bins - 1) / (kSpan * temperature), 3e38f);
    Found f = find_step(by_mass, by_mass ? 0 : u64(k), p, per, [&](float s, uint32_t at) { return bool(int(s > bs) | (int(s == bs) & int(at <= ba))); });
    const u64 target = f.target;
    const int step = f.bin;
    uint32_t prefix = 0;
    int shift = 32;  // key bits from `shift` up are fixed to prefix
    auto in = [&](uint32_t key, uint32_t at) {
      return kept(key, at, bk, ba) && (shift == 32 || (key >> shift) == prefix) && step_of(key_score(key), per) == step;
    };
    u64 before = f.before;
    int64_t size = f.size;
    while (size > a.cap && shift > 0) {
      const int next = shift - 8;
      // larger bytes first
      f = find(by_mass, 256, target, in, [&](float, uint32_t key, uint32_t) { return 255 - int((key >> next) & 255u); }, before);
      prefix = (prefix << 8) | uint32_t(255 - f.bin);
      shift = next;
      before = f.before;
      size = f.size;
    }
    if (size <= a.cap) {
      const bool with_draw = by_mass && shift == 32;
      if (with_draw) {
        *drawn = true;
        const float here = float(step) + 0x1p+23f;
        // without min-p the histogram has the w of all entries before the step
        need_mass = min_w > 0.f;
        if (!need_mass && rank == 0 && tid == 0) mass = float(before) * __int_as_float((127 - a.fix) << 23);
        draw([&](float s, uint32_t at) {
               return bool(int(s > -INFINITY) & int(step_up(s, per) < here) & (int(s > bs) | (int(s == bs) & int(at <= ba))));
             },
             [&](const float(&s)[kAhead][kG], int i) {
               bool any = false;
#pragma unroll
               for (int u = 0; u < kAhead; u++)
#pragma unroll
                 for (int j = 0; j < kG; j++) any |= fminf(step_up(s[u][j], per), last_up()) == here;
               if (!any) return;
#pragma unroll
               for (int u = 0; u < kAhead; u++)
#pragma unroll
                 for (int j = 0; j < kG; j++) {
                   const uint32_t key = order_key(s[u][j]), at = uint32_t(lo + i + u * threads * kG + j);
                   if (kept(key, at, bk, ba) && step_of(s[u][j], per) == step) list_add(key, at);
                 }
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
          u64 run = before;
          uint32_t last = 0;
          for (int j0 = 0; j0 < m; j0 += threads) {
            const int j = j0 + tid;
            u64 all;
            const float s = j < m ? key_score(uint32_t(sorted[j] >> 32)) : 0.f, w = j < m ? weight(s) : 0.f;
            const u64 ahead = run + scan(fixed(w), &all);
            if (j < m && ahead < target) {
              last = uint32_t(j) + 1;
              if (with_draw) list_consider(s, w, ~uint32_t(sorted[j]));
            }
            run += all;
          }
          last = block_max(last);
          e = sorted[last - 1];
        }
      }
      if (with_draw) {
        bound = e;
        return;
      }
      e = row_max(e);
      bound_key = uint32_t(e >> 32);
      bound_at = ~uint32_t(e);
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
               [&](uint32_t x, uint32_t at) { return x == key && at <= (x == bk ? ba : 0xffffffffu) && (above == 32 || (at >> above) == fixed_bits); },
               [&](float, uint32_t, uint32_t at) { return int((at >> next) & 255u); }, passed);
      ahead = (ahead << 8) | uint32_t(f.bin);
      passed = f.before;
    }
    bound_key = key;
    bound_at = ahead;
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
      if (before + all < u64(k)) return 1;  // fewer threads than k have an entry
      if (c && ahead < u64(k) && u64(k) <= ahead + c) found[0] = ahead, found[1] = u64(tid);
      __syncthreads();
      prefix = prefix << 8 | (255 - uint32_t(found[1]));
      before = uint32_t(found[0]);
      __syncthreads();
    }
    return prefix << 16;
  }

  // ---- the draw --------------------------------------------------------------------------

  // Whether the entry is so near the least that stays that recount has to look at it.
  template <bool kMinP, bool kMass = true>
  __device__ __forceinline__ bool consider(bool stays, float s, uint32_t at, float e) {
    const float x = (s - s_max) * exp2_per;
    if (kMass && need_mass) {
      const float w = stays ? fast_exp2(x) : 0.f;
      part += !kMinP || w >= min_w ? w : 0.f;
    }
    const bool in = stays && (!kMinP || x >= min_log2);
    const float key = in ? x - fast_log2(e) : -INFINITY;
    rough_second = fmaxf(rough_second, fminf(rough, key));
    const bool first = key > rough;
    rough = first ? key : rough;
    rough_at = first ? int32_t(at) : rough_at;
    return kMinP && in && x <= min_log2 + 2.f * kNear;
  }
  // The same of an entry whose w is known in full.
  __device__ __forceinline__ void list_consider(float s, float w, uint32_t at) {
    consider<true, false>(true, s, at, noise[at]);
    mass += w >= min_w ? w : 0.f;
  }
  // An entry that near the edge counts by its w in full, by which it is drawn or not, so that what is drawn is in the sum.
  __device__ __forceinline__ void recount(float s) {
    const float x = (s - s_max) * exp2_per;
    if (x >= min_log2 && x <= min_log2 + 2.f * kNear) {
      const float w = fast_exp2(x), full = weight(s);
      part += (full >= min_w ? full : 0.f) - (w >= min_w ? w : 0.f);
    }
  }
  // A turn's w to the sum, with the rounding kept: a thread may have thousands of turns, whose roundings
  // all go one way where scores are equal (1.6e-5 of the sum for 1.4 million entries of 512 threads).
  __device__ __forceinline__ void add_part() {
    const float2 had = turns[tid];
    const float more = part - had.y, sum = had.x + more;
    turns[tid] = make_float2(sum, (sum - had.x) - more);
    part = 0.f;
  }
  // An entry's key in full; 0 for one that min-p leaves out.
  __device__ __forceinline__ uint32_t exact(float s, float e) const {
    const float w = weight(s);
    return w >= min_w ? draw_key(w > 0.f ? __fdiv_rn(w, e) : 0.f) : 0;
  }
  // The thread's candidate in full; unsure where it has another one near or its w is near the least
  // that stays.
  __device__ __forceinline__ Drawn candidate(float s) const {
    Drawn d{0, 0xffffffffu, mass, order_key(rough_second)};
    if (rough_at >= 0) {
      d.key = exact(s, noise[rough_at]);
      if (d.key) d.at = uint32_t(rough_at);
      else d.unsure = order_key(rough);
    }
    return d;
  }
  __device__ __forceinline__ bool sure(const Drawn& d) const {
    return !d.unsure || key_score(d.unsure) < fast_log2(draw_value(d.key)) - kNear;
  }
  // Draws from the entries for which in(score, index) holds, which does for no masked score; also(scores,
  // i) sees all.
  template <typename In, typename Also>
  __device__ __forceinline__ void draw(In in, Also also) {
    if (min_w > 0.f) draw_by<true>(in, also);
    else draw_by<false>(in, also);
  }
  template <bool kMinP, typename In, typename Also>
  __device__ __forceinline__ void draw_by(In in, Also also) {
    const bool vector = a.noise_vector && skip % 4 == 0;
    turns[tid] = make_float2(0.f, 0.f);
    const float* const own = noise + lo;
    each_group([&](const float(&s)[kAhead][kG], int i) {
      bool stay[kAhead][kG];
      float e[kAhead][kG];
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        const int at = i + u * threads * kG;
        bool any = false;
#pragma unroll
        for (int j = 0; j < kG; j++) {
          stay[u][j] = in(s[u][j], uint32_t(lo + at + j));
          any |= stay[u][j];
        }
        if (vector && at >= 0 && at + kG <= count) {
          if (any) {
#pragma unroll
            for (int j = 0; j < kG; j += 4) {
              const float4 f = __ldcs(reinterpret_cast<const float4*>(own + at + j));
              e[u][j] = f.x, e[u][j + 1] = f.y, e[u][j + 2] = f.z, e[u][j + 3] = f.w;
            }
          }
        } else if (any) {
#pragma unroll
          for (int j = 0; j < kG; j++) e[u][j] = stay[u][j] ? own[at + j] : 1.f;
        }
      }
      also(s, i);
      bool near = false;
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        if (i + u * threads * kG >= count) break;
#pragma unroll
        for (int j = 0; j < kG; j++) near |= consider<kMinP>(stay[u][j], s[u][j], lo + i + u * threads * kG + j, e[u][j]);
      }
      if (kMinP && near) {  // rare: read again, so that nothing is kept for it
#pragma unroll 1
        for (int j = 0; j < kAhead * kG; j++) {
          const int at = i + j / kG * threads * kG + j % kG;
          if (at < 0 || at >= count) continue;
          const float v = value(global[at]);
          if (in(v, uint32_t(lo + at))) recount(v);
        }
      }
      if (need_mass) add_part();
    });
    mass += turns[tid].x;
  }
  // kept(score, index): what was drawn from.
  template <typename Kept>
  __device__ void finish(Kept kept_by, int32_t* index, float* logp) {
    const float s = rough_at >= 0 ? value(global[rough_at - lo]) : 0.f;  // of the row, not only of the slice
    Drawn got = row_best(candidate(s));
    if (!sure(got)) {
      // two candidates this close: every entry is computed in full (rows of equal scores and
      // noise; else about one row in 25,000)
      const u64 e = row_max(bound);
      Drawn all{0, 0xffffffffu, 0.f, 0};
      each([&](float v, int i) {
        const uint32_t at = uint32_t(lo + i);
        if (!(v > -INFINITY) || !kept_by(v, at, e)) return;
        const uint32_t key = exact(v, noise[at]);
        if (key > all.key) all.key = key, all.at = at;
      });
      const Drawn best = row_best(all);
      got.key = best.key, got.at = best.at;
    }
    if (rank == 0 && tid == 0) put(got, got.key ? value(global[int(got.at) - lo]) : 0.f, index, logp);
  }
  __device__ void put(const Drawn& d, float s, int32_t* index, float* logp) const {
    *index = d.key ? int32_t(d.at) : -1;  // none: no positive noise among what stays
    if (logp) *logp = d.key ? __fdiv_rn(s - s_max, temperature) - logf(d.mass) : -INFINITY;
  }
  // The first k of the list (m entries) hold all that stays: top-p and the draw on them, by the
  // row's first block.
  __device__ void finish_list(int k, int m, float p, int32_t* index, float* logp) {
    order(m);
    if (rank != 0) return;
    const int have = k < m ? k : m;
    u64 before = 0, total = 0, target = ~u64(0);
    const float s = tid < have ? key_score(uint32_t(sorted[tid] >> 32)) : 0.f;
    const float w = tid < have ? weight(s) : 0.f;
    const uint32_t at = tid < have ? ~uint32_t(sorted[tid]) : 0;
    if (p < 1.f) {
      before = scan(fixed(w), &total);
      target = p > 0.f ? share_of(total, p) : 1;
    }
    // one entry a thread: its candidate is sure
    if (tid < have && before < target) list_consider(s, w, at);
    const Drawn got = block_best(candidate(s));
    if (got.key ? tid < have && at == got.at : tid == 0) put(got, s, index, logp);
  }
};

// kFree: neither top-k nor top-p for any row.
template <typename T, int kThreads, bool kFree>
__global__ void __launch_bounds__(kThreads, 2048 / kThreads > 4 ? 4 : kThreads == 512 ? 2 : 1) sample_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int kG = Group<T>::kSize, kAhead = (kFree && kThreads < 1024 ? 16 : 8) / kG;  // 64 registers a thread
  __shared__ uint4 scratch[64], slots[2 * kMaxCluster];
  __shared__ u64 coarse[128], found[3];
  __shared__ int list_size[3];
  __shared__ float rest;
  Row<T, kAhead> r{cg::this_cluster(), a};
  r.tid = threadIdx.x, r.threads = kThreads, r.lane = r.tid & 31, r.warp = r.tid >> 5, r.warps = kThreads / 32;
  r.rank = int(r.cluster.block_rank()), r.blocks = int(r.cluster.num_blocks()), r.phase = r.turn = 0;
  r.scratch = scratch, r.slots = slots, r.found = found, r.list_size = list_size, r.coarse = coarse, r.rest = &rest;
  r.lists = 0, r.counted = false;
  if (threadIdx.x < 3) list_size[threadIdx.x] = 0;
  // a block's shared memory is written by others only when it is known to run; waited for after the loads
  if (r.blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  r.sums = reinterpret_cast<u64*>(smem);  // the first 256 steps; shares its memory with lacks
  r.lacks = reinterpret_cast<uint32_t*>(smem);
  r.counts = r.lacks + a.bins;
  r.sorted = r.sums;  // the histogram is done with when entries are ordered
  r.list = reinterpret_cast<u64*>(r.counts + (a.carry ? 2 : 1) * a.bins);
  r.turns = reinterpret_cast<float2*>(r.list + a.cap);
  r.data = reinterpret_cast<uint4*>(r.turns + kThreads);
  r.data_at = uint32_t(__cvta_generic_to_shared(r.data));
  r.counts_at = uint32_t(__cvta_generic_to_shared(r.counts)), r.lacks_at = uint32_t(__cvta_generic_to_shared(r.lacks));
  const int64_t row = blockIdx.x / unsigned(r.blocks);
  const int64_t lo = r.rank * a.slice, left = a.n - lo;
  r.lo = int(lo < a.n ? lo : a.n);
  r.count = int(left < 0 ? 0 : left < a.slice ? left : a.slice);
  r.global = static_cast<const T*>(a.scores) + row * a.row_stride + r.lo;
  r.skip = int(reinterpret_cast<uintptr_t>(r.global) % 16 / sizeof(T));
  r.groups = (r.skip + r.count + kG - 1) / kG;
  r.noise = a.noise + row * a.noise_stride;
  r.top_infinite = false;
  r.rough = r.rough_second = -INFINITY, r.rough_at = -1, r.need_mass = true, r.mass = r.part = 0.f, r.bound = 0;
  int32_t* index = a.index + row;
  float* logp = a.logp ? a.logp + row : nullptr;

  // scores once from memory: the thread's largest, and into shared memory
  float top = -INFINITY;
  for (int g = r.tid; g < r.groups; g += kThreads * 4) {
    Group<T> v[4];
#pragma unroll
    for (int u = 0; u < 4; u++) v[u] = r.fetch(g + u * kThreads);
#pragma unroll
    for (int u = 0; u < 4; u++) {
      if (g + u * kThreads < a.room) r.data[g + u * kThreads] = v[u].u;
#pragma unroll
      for (int j = 0; j < kG; j++) top = fmaxf(top, v[u].get(j));  // NaN is passed over
    }
  }
  r.held = r.groups < a.room ? r.groups : a.room;
  const uint32_t own = order_key(top);
  if (r.blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  const u64 top_key = r.row_max(r.block_max(own));
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
  r.min_log2 = r.min_w > 0.f ? fast_log2(r.min_w) - kNear : -INFINITY;
  const int64_t k = kFree ? 0 : a.top_k ? a.top_k[row] : a.top_k_all;
  const float p = kFree ? 1.f : a.top_p ? a.top_p[row] : a.top_p_all;
  __syncthreads();  // the scores are in shared memory

  if (!(r.temperature > 0.f)) {  // the largest score
    uint32_t first = 0;  // counted from the end, so that the lowest index is the largest
    r.each([&](float s, int i) {
      if (s == r.s_max) first = max(first, 0xffffffffu - uint32_t(r.lo + i));
    });
    const u64 at = r.row_max(r.block_max(first));
    if (r.rank == 0 && r.tid == 0) {
      *index = int32_t(0xffffffffu - uint32_t(at));
      if (logp) *logp = 0.f;
    }
    return;
  }
  if constexpr (kFree) {
    r.draw([](float s, uint32_t) { return s > -INFINITY; }, [](const auto&, int) {});
    r.finish([](float, uint32_t, u64) { return true; }, index, logp);
  } else {
    uint32_t bound_key = 0;
    uint32_t bound_at = 0xffffffffu;
    if (k > 0 && k < a.n) {
      if (k <= kThreads / 4) {
        // the k-th largest of one block's threads bounds the row's from below: the best of the blocks'
        const u64 least = r.row_max(r.floor_key(r.top_infinite ? (top == INFINITY ? order_key(0.f) : 0) : own, int(k)));
        const float low = least > 1 ? key_score(uint32_t(least)) : -INFINITY;
        r.each_group([&](const float(&s)[kAhead][kG], int i) {
#pragma unroll
          for (int u = 0; u < kAhead; u++) {
            float most = s[u][0];
#pragma unroll
            for (int j = 1; j < kG; j++) most = fmaxf(most, s[u][j]);
            if (!(most >= low)) continue;
#pragma unroll
            for (int j = 0; j < kG; j++)
              if (s[u][j] >= low && s[u][j] > -INFINITY) r.list_add(order_key(s[u][j]), r.lo + i + u * kThreads * kG + j);
          }
        });
        const int m = r.list_end();
        if (m <= a.cap) {
          r.finish_list(int(k), m, p, index, logp);
          r.sync();  // the list's size was read from the first block
          return;
        }
      }
      // a score is masked or counted: where fewer than k are left all of them stay
      uint32_t own_valid = 0;
      r.each([&](float s, int) { own_valid += s > -INFINITY; });
      u64 valid = 0, block_valid;
      r.scan(own_valid, &block_valid);
      if (r.blocks > 1) r.exchange(block_valid, [&](u64 x) { valid += x; });
      else valid = block_valid;
      if (u64(k) < valid) r.select(false, k, 0.f, bound_key, bound_at, nullptr);
    }
    bool drawn = false;
    if (p < 1.f) r.select(true, 0, fmaxf(p, 0.f), bound_key, bound_at, &drawn);
    const float bs = bound_key ? key_score(bound_key) : -INFINITY;
    if (!drawn)
      r.draw([&](float s, uint32_t at) { return bool(int(s > bs) | (int(s == bs) & int(at <= bound_at) & int(s > -INFINITY))); }, [](const auto&, int) {});
    r.finish(
        [&](float s, uint32_t at, u64 e) {  // e: the bound that a drawing selection left, 0 for none
          if (e) return r.kept(order_key(s), at, uint32_t(e >> 32), ~uint32_t(e));
          return s > bs || (s == bs && at <= bound_at);
        },
        index, logp);
  }
  // After the last exchange of a row no block reads another's memory: any may end first.
}

// How many clusters of each size, of blocks that fill an SM, run at the same time.
void clusters_at_once(int* fit) {
  for (int c = 1; c <= kMaxCluster; c++) {
    fit[c] = 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(c));
    cfg.blockDim = dim3(1024);
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(c);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    cfg.dynamicSmemBytes = kMostSmem;
    int n = 0;
    if (cudaFuncSetAttribute(sample_kernel<float, 1024, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) == cudaSuccess &&
        cudaOccupancyMaxActiveClusters(&n, sample_kernel<float, 1024, false>, &cfg) == cudaSuccess)
      fit[c] = n;
  }
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
  // Blocks of a row: as many as find an SM each at the same time (clusters that do not fit into
  // what is left of a group of SMs would wait) while a slice has 2048 entries.
  static std::once_flag once;
  static int fit[kMaxCluster + 1];
  std::call_once(once, [&] { clusters_at_once(fit); });
  int cluster = 1;
  for (int c = 2; c <= kMaxCluster; c++)
    if (rows <= fit[c] && a.n / c >= 2048) cluster = c;
  a.slice = ((a.n + cluster - 1) / cluster + 15) / 16 * 16;
  const bool wide = a.slice > 8192, crowd = int64_t(rows) * cluster > sms;
  // Shared memory of a block: all of an SM's, half where two blocks of 512 threads share one,
  // and what a short slice needs.
  a.bins = free ? 0 : !wide ? 512 : crowd ? 2048 : 4096;
  a.cap = free ? 0 : !wide ? 512 : crowd ? 1024 : 2048;
  const int threads = !wide ? 256 : crowd ? 512 : 1024;
  a.carry = !free && a.slice + 16 > int64_t(kCarryTurns) * threads * 8;
  size_t smem = size_t(a.bins) * (a.carry ? 12 : 8) + size_t(a.cap + threads) * 8;
  const size_t most = wide && !crowd ? kMostSmem : 110 * 1024;
  const size_t want = size_t(a.slice) * sizeof(T) + 16, room = most > smem ? most - smem : 0;
  a.room = int32_t((want < room ? want : room) / 16);
  smem += size_t(a.room) * 16;
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
  if (n > INT32_MAX - (1 << 20) || rows > (1 << 27)) return EMR_ERR_RANGE;
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
  a.noise_vector = reinterpret_cast<uintptr_t>(noise) % 16 == 0 && (rows == 1 || noise_stride % 4 == 0);
  const bool free = !top_k && !top_p && (top_k_all <= 0 || top_k_all >= n) && !(top_p_all < 1.f);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == EMR_F32) return plan<float>(a, rows, free, dev, sms, st);
  if (dtype == EMR_BF16) return plan<__nv_bfloat16>(a, rows, free, dev, sms, st);
  return plan<__half>(a, rows, free, dev, sms, st);
}
