// Log probabilities of given answers, entropies and best answers of rows of scores, and the gradient of the
// first two.
//
// With d_i = (s_i - max) / T, w_i = e^d_i and Z = sum w: logp_i = d_i - log Z, the entropy is log Z - (sum w d) / Z,
// and the gradient of a logp_t + b H is (a ([i = t] - p_i) - b p_i (log p_i + H)) / T. One pass over a row
// finds all three sums: a thread keeps its own maximum and its sums relative to that, and moves them when the
// maximum rises (rarely after its first entries); the threads', and the blocks', are joined in a fixed order. A
// gradient takes a second pass, which finds the row in L1 or L2 (those that are worked on at a time: of 349,524 float32 entries
// still, of 700,001 no longer), and writes once.
// Bound by memory where there are many rows: about seven operations and one exponential an entry, two of each in
// a gradient, are a good half of what an SM can do while an entry comes in. A row belongs to 8 threads or a warp where rows
// are short and many, to a block of 64 to 512, or to a cluster of up to 8 blocks where rows are few.
// The best k: the k-th largest of the threads' own maxima is at most the k-th largest score, so only threads whose
// maximum reaches it have their entries looked at again, by their warp, a lane for a group (about 25 of 128 threads for k =
// 20). What reaches it is collected and ordered. Rows with more such entries than the list holds (equal
// scores) find their k-th entry first, by a histogram of each byte of (score, index).
// Measured on the device: 4000 x 5460 float32 with its best 20 33 us (87 MB, 2.7 TB/s; 21.3 M instructions,
// 7 an entry for the sums and as many again for the search make 9.6 M of them, the rest, 2,900 a row, is what a row costs beside its entries; issue 57% of
// the time, the rest latency), without them 20; 24 x 349524 bfloat16 with its best 100 19 (six
// meetings of a cluster), gradients of 16000 x 340 bfloat16 10.9 (values alone 6.2) and of 512 x 87380 float32 with the entropy's 73 (358 MB, 4.9 TB/s), one
// row of 1364 with its best 5 4.5. Lists of more entries than a row has groups have it ordered as a whole: the best 100 of 8000 x 700 take 240 of
// bfloat16 and 81 of float32.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <float.h>

#include <mutex>
#include <type_traits>

#include "emr_score_rows.h"

namespace {

using namespace emr;
using namespace emr::rows;
typedef unsigned long long u64;

struct Args : Rows {
  const int32_t* target;
  float *logp, *entropy;
  const float *dlogp, *dentropy;
  float dlogp_all, dentropy_all;
  int32_t top;
  int32_t* top_index;
  float* top_logp;
};

// Shared memory of the search for the best.
template <int kTeam>
struct Best {
  static constexpr int kTeams = kTeam == 32 ? 8 : 1, kCap = kTeam == 32 ? 128 : kTeam == 64 ? 512 : kTeam == 512 ? 2048 : 1024;
  static constexpr int kTop = kTeam <= 64 ? 32 : kTeam == 128 ? 128 : EMR_MAX_TOP;
  u64 list[kTeams][kCap], sorted[kTeams][kTop], found[kTeams];
  alignas(16) uint32_t counts[kTeams][256];  // read 16 bytes at a time
  int size[kTeams][2];
  uint16_t who[kTeams][kTeam];
};

// The search for the best entries of a row, after its sums have been taken.
template <typename T, int kTeam>
struct Search : Row<T, kTeam> {
  typedef Row<T, kTeam> R;
  using R::blocks, R::cluster, R::exchange, R::floats, R::groups, R::head, R::kG, R::masked,
      R::kWarps, R::lane, R::lo, R::own, R::rank, R::row_sync, R::skip, R::team_max, R::team_sync, R::tid, R::value, R::warp, R::global;
  using R::R;

  template <typename V>
  __device__ __forceinline__ V* of_block(V* p, int r) { return blocks > 1 ? cluster.map_shared_rank(p, r) : p; }
  __device__ static u64 entry(uint32_t key, int at) { return (u64(key) << 32) | uint32_t(~at); }

  // The r-th largest key of a warp's threads, 0 where there are fewer.
  __device__ __forceinline__ uint32_t warp_kth(uint32_t key, int r) const {
    for (int i = 1; i < r; i++) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, key);
      if (lane == __ffs(int(__ballot_sync(0xffffffffu, key == top))) - 1) key = 0;
    }
    return __reduce_max_sync(0xffffffffu, key);
  }
  // A key that at least k of the row's threads' own largest reach, and few more: 1 where too few threads have one.
  __device__ uint32_t floor_key(int k, uint32_t* counts, u64* found) {
    const uint32_t mine = order_key(own.m);
    if (kTeam == 32) return max(warp_kth(mine, k), 1u);
    if (blocks == 1) {
      // every warp's r-th, r such that they have k together
      const int full = groups / 32 < kWarps ? groups / 32 : kWarps, r = full ? (k + full - 1) / full : 33;
      if (r <= 32) {
        const uint32_t low = ~team_max(warp < full ? ~warp_kth(mine, r) : 0u);
        if (low) return low;
      }
    } else {
      // the same over all blocks, of warps that have as many; then, as that is low, by equal steps from there to the
      // largest, so that little more than k are left
      struct Part {
        uint32_t top, low, warps, none;
      };
      const int r = (2 * k + kWarps * blocks - 1) / (kWarps * blocks);
      const uint32_t kth = r <= 32 ? warp_kth(mine, r) : 0u;
      Part all{0, 0xffffffffu, 0, 0};
      const uint32_t low_here = ~team_max(kth ? ~kth : 0u), top_here = team_max(mine);
      for (int b = tid; b < 256; b += kTeam) counts[b] = 0;
      const uint32_t warps_here = __syncthreads_count(kth && lane == 0);
      exchange(Part{top_here, low_here, warps_here, 0}, [&](const Part& x) {
        all.top = max(all.top, x.top), all.low = min(all.low, x.low), all.warps += x.warps;
      });
      if (int64_t(all.warps) * r >= k) {
        const float top = key_score(all.top), span = top - key_score(all.low);
        const float steps = span > 0.f ? fminf(255.f / span, 3e38f) : 0.f;
        if (mine >= all.low) atomicAdd(counts + min(255, int((top - key_score(mine)) * steps)), 1u);
        row_sync();
        if (warp == 0) {
          uint32_t c[8] = {}, sum = 0;
          for (int b = 0; b < blocks; b++) {
            const uint4* const of = reinterpret_cast<const uint4*>(of_block(counts, b)) + lane * 2;
            const uint4 x = of[0], y = of[1];
            c[0] += x.x, c[1] += x.y, c[2] += x.z, c[3] += x.w, c[4] += y.x, c[5] += y.y, c[6] += y.z, c[7] += y.w;
          }
#pragma unroll
          for (int j = 0; j < 8; j++) sum += c[j];
          uint32_t before = sum;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += x;
          }
          before -= sum;
#pragma unroll
          for (int j = 0; j < 8; j++) {
            if (before < uint32_t(k) && uint32_t(k) <= before + c[j]) *found = u64(lane * 8 + j);
            before += c[j];
          }
        }
        team_sync();
        const int step = int(*found);
        // the least key of that step: keys and steps fall together
        uint32_t least = all.low, past = all.top;
        while (least < past) {
          const uint32_t mid = least + (past - least) / 2;
          if (min(255, int((top - key_score(mid)) * steps)) <= step) past = mid;
          else least = mid + 1;
        }
        return max(least, 1u);  // the counts are written again only after the next barrier of the row
      }
    }
    // the k-th of a block's threads, bit by bit, and the best of the blocks' own
    uint32_t low = 0;
    for (int bit = 31; bit >= 12; bit--) {
      const uint32_t more = low | 1u << bit;
      if (__syncthreads_count(mine >= more) >= k) low = more;
    }
    if (blocks > 1) {
      const uint32_t part = low;
      exchange(part, [&](uint32_t x) { low = max(low, x); });
    }
    return max(low, 1u);
  }
  // The entries from `least` on to the list of the row's first block (dropped past its room, but counted): the groups of
  // the threads whose own largest is one of them are shared out over their warp.
  __device__ int collect(u64 least, Best<kTeam>& b, int team, int round) {
    const uint32_t low = uint32_t(least >> 32);
    const float low_score = low > 1 ? key_score(low) : -FLT_MAX;
    const bool hit = order_key(own.m) >= low;
    const uint32_t hits = __ballot_sync(0xffffffffu, hit);
    uint16_t* const who = b.who[team] + warp * 32;
    if (hit) who[__popc(hits & ((1u << lane) - 1))] = uint16_t(tid);
    __syncwarp();
    u64* const to = of_block(b.list[team], 0);
    int* const places = of_block(b.size[team] + round, 0);
    const unsigned each_has = unsigned(groups + kTeam - 1) / kTeam;  // groups of a thread at most, the first of all as the last of one
    for (unsigned i = lane; i < __popc(hits) * each_has; i += 32) {
      const unsigned h = i / each_has;
      const int at = head + who[h] + int(i - h * each_has) * kTeam, g = at == groups ? 0 : at;
      if (at >= groups + head) continue;
      const Group<T> v = masked(g);
      uint32_t reach = 0;
#pragma unroll
      for (int j = 0; j < kG; j++) reach |= uint32_t(v.get(j) >= low_score) << j;
      for (; reach; reach &= reach - 1) {  // few: read again
        const int from = g * kG - skip + __ffs(int(reach)) - 1;
        const u64 e = entry(order_key(value(global[from])), lo + from);
        if (e < least) continue;
        const int place = atomicAdd(places, 1);
        if (place < b.kCap) to[place] = e;
      }
    }
    row_sync();
    return *places;
  }
  // The k-th entry in order, of a row that has as many, or one after it and before the next.
  __device__ u64 kth(int k, uint32_t* counts, u64* found) {
    u64 prefix = 0;
    for (int shift = 56;; shift -= 8) {
      for (int b = tid; b < 256; b += kTeam) counts[b] = 0;
      team_sync();
      int bin = -1;  // equal entries that follow each other are counted together
      uint32_t run = 0;
      for (int g = tid; g < groups; g += kTeam) {
        const Group<T> v = masked(g);
#pragma unroll
        for (int j = 0; j < kG; j++) {
          const uint32_t key = order_key(v.get(j));
          const u64 e = entry(key, lo + g * kG - skip + j);
          if (!key || (shift < 56 && e >> (shift + 8) != prefix)) continue;
          const int b = 255 - int((e >> shift) & 255u);
          if (b != bin) {
            if (run) atomicAdd(counts + bin, run);
            bin = b, run = 0;
          }
          run++;
        }
      }
      if (run) atomicAdd(counts + bin, run);
      row_sync();
      // the step in which the k-th lies: a lane has eight, of all blocks
      if (warp == 0) {
        uint32_t c[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          c[j] = 0;
          for (int r = 0; r < blocks; r++) c[j] += of_block(counts, r)[lane * 8 + j];
          sum += c[j];
        }
        uint32_t before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += x;
        }
        before -= sum;
        if (before < uint32_t(k) && uint32_t(k) <= before + sum) {
          for (int j = 0; j < 8; j++) {
            if (before < uint32_t(k) && uint32_t(k) <= before + c[j])
              *found = (u64(before) << 32) | (uint32_t(lane * 8 + j) << 1) | uint32_t(before + c[j] == uint32_t(k));
            before += c[j];
          }
        }
      }
      team_sync();
      const u64 f = *found;
      k -= int(f >> 32);
      prefix = prefix << 8 | (255 - (uint32_t(f) >> 1));
      row_sync();  // read before it is written again, and by the other blocks
      if (f & 1 || shift == 0) return prefix << shift;
    }
  }
  // The list's m entries in order, in `sorted` of the row's first block, as far as it holds them: an entry's place is
  // the number of larger ones. Of more than 64 entries each 32 are sorted by a warp, and counted by bisection (about 208
  // entries for the best 100 of 5460: 4000 rows 88 -> 73 us).
  __device__ void order(int m, u64* list, u64* sorted, int room) {
    if (rank == 0) {
      const bool parts = m > 64;
      if (parts) {
        for (int c = warp * 32; c < m; c += kWarps * 32) {
          u64 e = c + lane < m ? list[c + lane] : 0;
#pragma unroll
          for (int size = 2; size <= 32; size *= 2)
#pragma unroll
            for (int apart = size / 2; apart; apart /= 2) {
              const u64 other = __shfl_xor_sync(0xffffffffu, e, apart);
              const bool first = !(lane & apart), down = !(lane & size) || size == 32;
              e = (other > e) == (first == down) ? other : e;
            }
          list[c + lane] = e;
        }
        team_sync();
      }
      for (int j = tid; j < m; j += kTeam) {
        const u64 e = list[j];
        int larger = 0;
        if (!parts) {
#pragma unroll 8
          for (int i = 0; i < m; i++) larger += list[i] > e;
        } else {
          larger = j & 31;
          for (int c = 0; c < m; c += 32) {
            if (c == (j & ~31)) continue;
            int n = 0;
#pragma unroll
            for (int step = 16; step; step /= 2) n += list[c + n + step - 1] > e ? step : 0;
            larger += n + (list[c + n] > e);
          }
        }
        if (larger < room) sorted[larger] = e;
      }
    }
    team_sync();
  }
  // The best k of the row, in b.sorted of the row's first block; their number.
  __device__ int best(int k, Best<kTeam>& b, int team) {
    int m = collect(u64(floor_key(k, b.counts[team], b.found + team)) << 32, b, team, 0);
    if (m > b.kCap) m = collect(kth(k, b.counts[team], b.found + team), b, team, 1);
    order(m, b.list[team], b.sorted[team], b.kTop);
    return m < k ? m : k;
  }

};

// Entries of a gradient: w (k1 d + k0), and the same everywhere.
struct Slope {
  float m, per, k1, k0;
  __device__ __forceinline__ float2 operator()(float s0, float s1) const {
    const float2 d = far2(s0, s1, m, per);
    return mul2(make_float2(fast_exp2(d.x), fast_exp2(d.y)), fma2(d, make_float2(k1, k1), make_float2(k0, k0)));
  }
};
struct Same {
  float v;
  __device__ __forceinline__ float2 operator()(float, float) const { return make_float2(v, v); }
};

// What a kernel is asked for besides the sums.
enum Ask { kSums, kTop, kGradient };

template <typename T, int kTeam, int kAsk>
__global__ void __launch_bounds__(kTeam <= 32 ? 256 : kTeam, kTeam == 512 ? 2 : kTeam == 64 ? 20 : kTeam == 128 ? 10 : 4) log_probs_kernel(const __grid_constant__ Args a) {
  constexpr int kRows = kTeam <= 32 ? 256 / kTeam : 1;  // of a block
  __shared__ uint4 scratch[kTeam <= 32 ? 1 : 64], slots[kTeam == 512 ? 2 * kMaxCluster : 1];
  __shared__ std::conditional_t<kAsk == kTop, Best<kTeam>, uint32_t> best;
  const int team = kTeam <= 32 ? threadIdx.x / kTeam : 0;
  int64_t row = kTeam < 512 ? int64_t(blockIdx.x) * kRows + team : int64_t(blockIdx.x / cg::this_cluster().num_blocks());
  const bool there = row < a.rows;
  if (kTeam == 32 && !there) return;
  if (kTeam < 32 && !there) row = a.rows - 1;  // a team without a row takes the last one's and writes nothing
  Search<T, kTeam> r(a, row, scratch, slots);
  if constexpr (kAsk == kTop) {
    if (r.tid < 2) best.size[team][r.tid] = 0;
  }
  // a block's shared memory is written by others only when it is known to run; waited for after the pass
  if (r.blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  const float temperature = a.temperature ? a.temperature[row] : a.temperature_all;
  const bool greedy = !(temperature > 0.f);
  const int64_t target = a.target ? a.target[row] : -1;
  const float dlogp = kAsk == kGradient ? (a.dlogp ? a.dlogp[row] : a.dlogp_all) : 0.f;
  const float dentropy = kAsk == kGradient ? (a.dentropy ? a.dentropy[row] : a.dentropy_all) : 0.f;
  r.per = greedy ? 0.f : fminf(kLog2E / temperature, 3e38f);
  r.asks = kAsk == kGradient;

  Stat all;
  for (bool again = false;; again = true) {
    r.sum_up();
    if (!again && r.blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    all = r.total();
    if (all.m < INFINITY) break;
    r.top_infinite = true;
  }
  const bool empty = all.m == -INFINITY;
  // what is written for the row, and by whom; the others need no logarithm
  const bool tells = r.rank == 0 && (r.tid < (kAsk == kTop ? max(a.top, 1) : 1));
  const bool uncertain = kAsk == kGradient && dentropy != 0.f;
  float log_z = 0.f, entropy = 0.f;
  if (tells || uncertain) {
    log_z = logf(all.s);
    entropy = empty || greedy ? 0.f : fmaxf(log_z - kLn2 * __fdiv_rn(all.e, all.s), 0.f);
  }
  const auto log_prob = [&](float s) { return s - all.m > -INFINITY ? __fdiv_rn(s - all.m, temperature) - log_z : -INFINITY; };

  const int64_t first = greedy && !empty && a.logp ? r.first(all.m) : -1;
  if constexpr (kAsk == kTop) {
    const int got = empty ? 0 : r.best(a.top, best, team);
    if (r.rank == 0) {
      for (int j = r.tid; j < a.top; j += kTeam) {
        const u64 e = j < got ? best.sorted[team][j] : 0;
        const int64_t at = row * a.top + j;
        if (a.top_index) a.top_index[at] = e ? int32_t(~uint32_t(e)) : -1;
        if (a.top_logp) a.top_logp[at] = !e ? -INFINITY : greedy ? (j == 0 ? 0.f : -INFINITY) : log_prob(key_score(uint32_t(e >> 32)));
      }
    }
    if (r.blocks > 1) r.cluster.sync();  // the list's size was read from the first block
  }
  if (r.rank == 0 && r.tid == 0 && there) {
    if (a.logp) {
      const T* const scores = static_cast<const T*>(a.scores) + row * a.row_stride;
      float v = 0.f;
      if (target >= a.n) v = NAN;
      else if (target >= 0) v = greedy ? (target == first ? 0.f : -INFINITY) : log_prob(r.value(scores[target]));
      a.logp[row] = v;
    }
    if (a.entropy) a.entropy[row] = entropy;
  }
  if constexpr (kAsk == kGradient) {
    // w (k1 d + k0), with p = w / Z and log p = d ln 2 - log Z
    const float per_t = greedy ? 0.f : fminf(__fdiv_rn(1.f, temperature), 3e38f);
    const float da = target < 0 ? 0.f : target >= a.n ? NAN : dlogp;
    const float inverse = empty ? 0.f : __fdiv_rn(-per_t, all.s), m = empty ? 0.f : all.m, hit = da * per_t;
    const float k1 = inverse * dentropy * kLn2, k0 = inverse * (uncertain ? fmaf(dentropy, entropy - log_z, da) : da);
    if (kTeam < 32 && !there) return;
    const typename Row<T, kTeam>::Out o = r.out(a, row);
    r.asks = false;
    if (empty || isnan(da + dentropy)) {
      r.put(o, Same{empty && !isnan(da + dentropy) ? 0.f : NAN});
      return;
    }
    r.put(o, Slope{m, r.per, k1, k0});
    // once more where the answer stands
    r.team_sync();
    if (r.tid == 0 && target >= r.lo && target - r.lo < r.count) {
      const int i = int(target - r.lo);
      const float s = r.value(r.global[i]);
      if (s > -INFINITY) store_scalar(o.p, o.dtype, i, Slope{m, r.per, k1, k0}(s, s).x + hit);
    }
  }
}

// The same for every kind of call, so that all of them sum a row in the same order.
const int* fits() {
  static std::once_flag once;
  static int fit[kMaxCluster + 1];
  std::call_once(once, [&] { clusters_at_once(log_probs_kernel<float, 512, kTop>, 512, fit); });
  return fit;
}

template <typename T, int kAsk>
emr_status log_probs(Args a, int sms, cudaStream_t st) {
  // Longer lists by more threads, as each part of 32 entries is a warp's; but rows that are many keep an SM busy with 128. By 128 and
  // 256 threads, in us: 40 best of 4000 x 5460 float32 41 and 54, of 1000 x 2000 9.6 and 12; 100 best of 16000 x 340 163 and 257, 4000 x
  // 5460 74 and 75, 2000 x 8000 59 and 50, 700 x 5460 25 and 19.
  const int longer = a.top <= 64 || (a.top <= Best<128>::kTop && a.rows >= 24 * sms) ? 128 : 256;
  const int least = kAsk != kTop ? 8 : a.top <= Best<32>::kTop ? 32 : longer;
  int cluster;
  const int team = plan(a, least, sizeof(T), sms, fits(), &cluster);
  if constexpr (kAsk != kTop) {
    if (team == 8) return launch_rows(log_probs_kernel<T, 8, kAsk>, a, team, cluster, st);
  }
  return team == 32    ? launch_rows(log_probs_kernel<T, 32, kAsk>, a, team, cluster, st)
         : team == 64  ? launch_rows(log_probs_kernel<T, 64, kAsk>, a, team, cluster, st)
         : team == 128 ? launch_rows(log_probs_kernel<T, 128, kAsk>, a, team, cluster, st)
         : team == 256 ? launch_rows(log_probs_kernel<T, 256, kAsk>, a, team, cluster, st)
                       : launch_rows(log_probs_kernel<T, 512, kAsk>, a, team, cluster, st);
}
template <int kAsk>
emr_status log_probs(const Args& a, int dtype, int sms, cudaStream_t st) {
  if (dtype == EMR_F32) return log_probs<float, kAsk>(a, sms, st);
  if (dtype == EMR_BF16) return log_probs<__nv_bfloat16, kAsk>(a, sms, st);
  return log_probs<__half, kAsk>(a, sms, st);
}

}  // namespace

extern "C" emr_status emr_log_probs(const void* scores, int32_t dtype, int32_t rows, int64_t n, int64_t row_stride,
                                    const int32_t* target, const float* temperature, float temperature_all, int32_t top, float* logp,
                                    float* entropy, int32_t* top_index, float* top_logp, void* stream) {
  const emr_status ok = check_scores(scores, dtype, rows, n, row_stride);
  if (ok != EMR_OK) return ok;
  if (top < 0 || (logp && !target) || !aligned(target, 4) || !aligned(temperature, 4) || !aligned(logp, 4) || !aligned(entropy, 4) ||
      !aligned(top_index, 4) || !aligned(top_logp, 4) || (!logp && !entropy && !(top && (top_index || top_logp))))
    return EMR_ERR_ARG;
  if (top > EMR_MAX_TOP) return EMR_ERR_RANGE;
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  Args a{};
  a.scores = scores, a.n = n, a.row_stride = row_stride, a.rows = rows;
  a.temperature = temperature, a.temperature_all = temperature_all;
  a.target = target, a.logp = logp, a.entropy = entropy;
  a.top = top, a.top_index = top_index, a.top_logp = top_logp;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return top && (top_index || top_logp) ? log_probs<kTop>(a, dtype, sms, st) : log_probs<kSums>(a, dtype, sms, st);
}

extern "C" emr_status emr_log_probs_grad(const void* scores, int32_t dtype, int32_t rows, int64_t n, int64_t row_stride,
                                         const int32_t* target, const float* temperature, float temperature_all, const float* dlogp,
                                         float dlogp_all, const float* dentropy, float dentropy_all, float* logp, float* entropy,
                                         void* dscores, int32_t d_dtype, int64_t d_stride, void* stream) {
  const emr_status ok = check_scores(scores, dtype, rows, n, row_stride);
  if (ok != EMR_OK) return ok;
  if (!target || !dscores || !dtype_ok(d_dtype) || d_stride < n || !aligned(dscores, dtype_bytes(d_dtype)) || !aligned(target, 4) ||
      !aligned(temperature, 4) || !aligned(dlogp, 4) || !aligned(dentropy, 4) || !aligned(logp, 4) || !aligned(entropy, 4) ||
      overlap(scores, (rows - 1) * row_stride + n, dtype_bytes(dtype), dscores, (rows - 1) * d_stride + n, dtype_bytes(d_dtype)))
    return EMR_ERR_ARG;
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  Args a{};
  a.scores = scores, a.n = n, a.row_stride = row_stride, a.rows = rows;
  a.temperature = temperature, a.temperature_all = temperature_all;
  a.target = target, a.logp = logp, a.entropy = entropy;
  a.dlogp = dlogp, a.dlogp_all = dlogp_all, a.dentropy = dentropy, a.dentropy_all = dentropy_all;
  a.dscores = dscores, a.d_dtype = d_dtype, a.d_stride = d_stride;
  return log_probs<kGradient>(a, dtype, sms, static_cast<cudaStream_t>(stream));
}
