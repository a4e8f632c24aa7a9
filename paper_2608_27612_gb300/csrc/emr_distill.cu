// Distillation: the loss of rows of scores against the best answers of a teacher, and its gradient.
//
// The teacher's record of a row is a list of k (entry i_j, log probability l_j). With t_j = e^l_j, or softmax(l) where
// the list stands for all of the teacher, and p = softmax(s / T): the loss is sum t_j (log t_j - log p_i_j), and where what the
// list leaves over counts as one more answer ("tail"), plus t_r (log t_r - log p_r), with t_r = 1 - sum t_j and p_r the
// sum of p over the rest, the entries that are not listed. dL/ds_i is M p_i - t_i for a listed entry, M = sum t + t_r, and
// for one of the rest, e_i (M / Z - t_r / z_r) = e_i / z_r (p_r sum t - t_r p_l), p_l being 1 - p_r: without a small difference of
// sums near 1, but for t_r itself, whose sum is kept in two parts (split_exp). For the same reason the rest has sums of its own, in which listed entries are left out by a bit for
// each entry (one byte of shared memory is looked at for 8 of them), and its own maximum, so that a
// rest of 1e-30 has a softmax like any other.
// As for log probabilities, one pass over the row for the sums and, for the gradient, a second one that finds it in
// L1 or L2 (where the rows that are worked on at a time fit there) and writes once; listed entries are written over after it, k of them. Bound by memory for many rows; for
// few, by the chain list - scores of its entries - bits - pass - sums.
// Measured on the device: 2000 x 5460 bfloat16 with lists of 50 19 us (44 MB; a row costs 750 instructions a warp beside its
// entries), 1000 x 87380 float16 with 64 79 (350 MB, 4.4 TB/s; issue 55%, exponentials 48% of their unit), 250 x 1364 float32
// with 16 6.2; the loss alone 11.6, 53 and 5.5.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <mutex>

#include "emr_score_rows.h"

namespace {

using namespace emr;
using namespace emr::rows;

struct Args : Rows {
  const int32_t* index;
  const void* teacher;
  int32_t teacher_dtype, k, tail;
  const float* dloss;
  float dloss_all;
  float* loss;
};

// Shared memory of a row's list, and a byte for each group of a piece of the slice, a bit of it for each entry.
template <int kTeam>
struct List {
  static constexpr int kTeams = kTeam == 32 ? 8 : 1, kMost = kTeam == 32 ? 64 : EMR_MAX_TOP;
  static constexpr int kBytes = kTeam == 32 ? 288 : kTeam < 512 ? 2080 : 16384;  // of groups of a piece; rows of less than a cluster are one piece
  int at[kTeams][kMost];                                           // -1: none
  float l[kTeams][kMost], t[kTeams][kMost], s[kTeams][kMost];
  uint32_t bits[kTeams][kBytes / 4];
  int twice[kTeams];  // an entry is listed more than once
};

// Sums of entries that are not listed.
template <typename R>
struct AddRest {
  R& r;
  const uint8_t* listed;
  template <typename G, int kN>
  __device__ __forceinline__ void operator()(const G (&v)[kN], int g) {
    G x[kN];
#pragma unroll
    for (int u = 0; u < kN; u++) {
      x[u] = v[u];
      const uint32_t l = listed[g + u * R::kTeamSize];
      if (l) {
#pragma unroll
        for (int j = 0; j < R::kG; j++)
          if (l >> j & 1) x[u].mask(j);
      }
    }
    r.template add<false>(x);
  }
};
// An entry of the rest in the gradient.
struct Slope {
  float m, per, coef;
  __device__ __forceinline__ float2 operator()(float s0, float s1) const {
    const float2 d = far2(s0, s1, m, per);
    return mul2(make_float2(fast_exp2(d.x), fast_exp2(d.y)), make_float2(coef, coef));
  }
};

__device__ __forceinline__ float load_scalar(const void* p, int dtype, int64_t i) {
  if (dtype == EMR_F32) return static_cast<const float*>(p)[i];
  if (dtype == EMR_BF16) return float(static_cast<const __nv_bfloat16*>(p)[i]);
  return float(static_cast<const __half*>(p)[i]);
}

// A teacher's probability e^l, all of it and as high + low. What a list leaves over, 1 - sum t, is often 1e-5 and less, of 32-bit values
// that are each off by 2^-25 and more; high is a multiple of 2^-22, sums of which are exact up to 4 (beyond that nothing is left over), and
// low the rest of e^l to 6e-13 e^l: sums of up to 256 parts of at most 2^-23 are off by at most 12 2^-24 2^-15 = 2.2e-11.
// e^l = 2^(k / 2) e^r, |r| <= ln 2 / 4, with k ln 2 / 2 taken off in two parts (Cody and Waite) and the series r + r^2 (12 + 4 r + r^2) / 24 in two
// floats a value (Dekker's sums and products), from r^5 on in one: 0.5 us of 2000 lists of 50, where exp in 64 bits takes 4.4.
struct Parts {
  float all, high, low;
};
__device__ __forceinline__ Parts split_exp(float l) {
  const float all = expf(l);
  if (!(all < 2.f)) return {all, all, 0.f};
  const float high = __fsub_rn(__fadd_rn(all, 3.f), 3.f);
  if (l < -40.f) return {all, 0.f, all};
  const float k = rintf(l * (2.f * kLog2E));
  const float r0 = __fmaf_rn(-k, 0x1.62e4p-2f, l), r = __fmaf_rn(-k, 0x1.7f7d1cp-21f, r0), r_low = __fmaf_rn(-k, 0x1.7f7d1cp-21f, r0 - r);
  const float tail = __fmaf_rn(__fmaf_rn(__fmaf_rn(r, 1.f / 40320.f, 1.f / 5040.f), r, 1.f / 720.f), r, 1.f / 120.f);
  const float s = __fmul_rn(r, r), s_low = __fmaf_rn(r, r, -s);
  const float v = __fmaf_rn(4.f, r, 12.f), v_low = __fmaf_rn(4.f, r, 12.f - v);
  const float w = __fadd_rn(v, s), w_low = ((v - w) + s) + (v_low + s_low);
  const float p = __fmul_rn(s, w), p_low = __fmaf_rn(s, w, -p) + __fmaf_rn(s, w_low, s_low * w);
  constexpr float kPart = 1.f / 24.f, kPartLow = float(1. / 24. - double(kPart));
  const float q = __fmul_rn(p, kPart), q_low = __fmaf_rn(p, kPart, -q) + __fmaf_rn(p, kPartLow, p_low * kPart);
  const float a = __fadd_rn(1.f, r), a_low = r - (a - 1.f);
  const float b = __fadd_rn(a, q), b_low = q - (b - a);
  const float rest = __fmaf_rn(tail, s * s * r, q_low) + __fmaf_rn(r_low, b, a_low + b_low);
  constexpr float kRoot = 1.41421356f, kRootLow = float(1.41421356237309504880 - double(kRoot));
  const int n = int(k);
  const float root = n & 1 ? kRoot : 1.f, root_low = n & 1 ? kRootLow : 0.f;
  const float e = __fmul_rn(b, root), e_low = __fmaf_rn(b, root, -e) + __fmaf_rn(b, root_low, rest * root);
  const float scale = __uint_as_float(uint32_t((n >> 1) + 127) << 23);
  return {all, high, __fmaf_rn(e, scale, -high) + e_low * scale};
}

template <typename T, int kTeam>
__global__ void __launch_bounds__(kTeam == 32 ? 256 : kTeam, kTeam == 512 ? 2 : kTeam == 64 ? 16 : kTeam == 128 ? 8 : 4) distill_kernel(const __grid_constant__ Args a) {
  typedef Row<T, kTeam> R;
  constexpr int kG = R::kG, kPiece = List<kTeam>::kBytes;
  __shared__ uint4 scratch[kTeam == 32 ? 1 : 64], slots[kTeam == 512 ? 2 * kMaxCluster : 1];
  __shared__ List<kTeam> lists;
  const int team = kTeam == 32 ? threadIdx.x >> 5 : 0;
  const int64_t row = kTeam == 32 ? int64_t(blockIdx.x) * 8 + team : kTeam < 512 ? int64_t(blockIdx.x) : int64_t(blockIdx.x / cg::this_cluster().num_blocks());
  if (kTeam == 32 && row >= a.rows) return;
  R r(a, row, scratch, slots);
  if (r.blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  int* const at = lists.at[team];
  float *const l = lists.l[team], *const t = lists.t[team], *const s = lists.s[team];
  uint32_t* const bits = lists.bits[team];
  const T* const scores = static_cast<const T*>(a.scores) + row * a.row_stride;
  const float temperature = a.temperature ? a.temperature[row] : a.temperature_all;
  const bool heat = temperature > 0.f;
  r.per = heat ? fminf(kLog2E / temperature, 3e38f) : 0.f;

  r.ahead();
  r.asks = a.dscores != nullptr;
  const auto clear = [&](int groups) {
    for (int w = r.tid; w < (groups + 3) / 4; w += kTeam) bits[w] = 0;
  };
  const auto mark = [&](int from, int past) {
    for (int j = r.tid; j < a.k; j += kTeam) {
      if (at[j] < r.lo || at[j] - r.lo >= r.count) continue;
      const int i = at[j] - r.lo + r.skip, b = i / kG - from;
      if (b < 0 || b >= past - from) continue;
      const uint32_t bit = 1u << (b % 4 * 8 + i % kG);
      if (atomicOr(bits + b / 4, bit) & bit) lists.twice[team] = 1;
    }
  };
  const int first_piece = min(r.groups, kPiece);
  clear(first_piece);

  // the list; what cannot be told from it turns the row into NaN
  float wrong = heat ? 0.f : NAN;
  uint32_t l_key = 0, s_key = 0;
  for (int j = r.tid; j < a.k; j += kTeam) {
    const int i = a.index[row * a.k + j];
    const float v = load_scalar(a.teacher, a.teacher_dtype, row * a.k + j);
    const bool in = i >= 0 && i < a.n;
    if (i >= a.n || (in && isnan(v))) wrong = NAN;
    at[j] = in ? i : -1;
    l[j] = in ? v : -INFINITY;
    s[j] = in ? float(scores[i]) : -INFINITY;
    l_key = max(l_key, order_key(l[j]));
    s_key = max(s_key, order_key(s[j]));
  }
  if (r.tid == 0) lists.twice[team] = 0;
  s_key = r.team_max(s_key);
  if (kTeam == 32) r.team_sync();
  mark(0, first_piece);
  float m_listed = s_key ? key_score(s_key) : -INFINITY;
  float l_max = 0.f;
  if (!a.tail) {
    l_key = r.team_max(l_key);
    l_max = l_key ? key_score(l_key) : 0.f;
  }
  const auto weight = [&](int j, float m) { return s[j] > -INFINITY ? fast_exp2(fmaxf((s[j] - m) * r.per, kFar)) : 0.f; };
  // sums of t, in two parts where 1 - sum t is wanted, and of the listed entries' w relative to their own maximum if each stands there once
  float part = 0.f, low = 0.f, z_first = 0.f;
  for (int j = r.tid; j < a.k; j += kTeam) {
    if (a.tail) {
      Parts e = split_exp(l[j]);
      t[j] = e.all, part += e.high, low += e.low;
    } else {
      part += t[j] = expf(l[j] - l_max);
    }
    if (r.blocks == 1) z_first += weight(j, m_listed);
  }
  const float3 sums = r.team_sum(make_float3(part + wrong, low, z_first));
  if (kTeam == 32) r.team_sync();  // a block's sums are barriers
  z_first = sums.z;
  const float t_sum = !a.tail && sums.x > 0.f ? 1.f : sums.x + sums.y;
  float t_scale = 1.f, l_base = 0.f;  // log t_j = l_j - l_base
  if (!a.tail && sums.x > 0.f) t_scale = __fdiv_rn(1.f, sums.x), l_base = l_max + logf(sums.x);
  const float left = (1.f - sums.x) - sums.y;  // the difference is exact, so this is rounded once

  // the rest's sums
  Stat rest;
  bool again = false;
  for (;; again = true) {
    r.begin();
    for (int from = 0; from < r.groups; from += kPiece) {
      const int past = r.groups - from < kPiece ? r.groups : from + kPiece;
      if (from || again) {
        r.team_sync();
        clear(past - from);
        r.team_sync();
        mark(from, past);
        r.team_sync();
      }
      AddRest<R> add{r, reinterpret_cast<const uint8_t*>(bits) - from};
      r.each(add, from ? from : r.head, past, from == 0);
    }
    if (!again && r.blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // the row's other blocks run
    rest = r.total();
    if (rest.m < INFINITY && m_listed < INFINITY) break;
    m_listed = m_listed == INFINITY ? 0.f : -INFINITY;
    r.top_infinite = true;
    r.team_sync();
    for (int j = r.tid; j < a.k; j += kTeam) s[j] = s[j] == INFINITY ? 0.f : -INFINITY;
    if (r.tid == 0) lists.twice[team] = 0;
  }
  const bool twice = lists.twice[team] != 0;
  const float m = fmaxf(rest.m, m_listed);
  const bool empty = m == -INFINITY, has_rest = rest.m > -INFINITY;
  // listed entries of the slice, each once
  const auto mine = [&](int j) {
    if (at[j] < r.lo || at[j] - r.lo >= r.count) return false;
    if (twice)
      for (int i = 0; i < j; i++)
        if (at[i] == at[j]) return false;
    return true;
  };
  float z_listed;
  if (r.blocks == 1 && !twice && !again) {
    z_listed = z_first * (s_key ? fast_exp2(fmaxf((m_listed - m) * r.per, kFar)) : 0.f);
  } else {
    part = 0.f;
    for (int j = r.tid; j < a.k; j += kTeam)
      if (mine(j)) part += weight(j, m);
    z_listed = r.team_sum(make_float2(part, 0.f)).x;
  }
  if (r.blocks > 1) {
    const float own = z_listed;
    z_listed = 0.f;
    r.exchange(own, [&](float x) { z_listed += x; });
  }
  const float z_rest = has_rest ? rest.s * fast_exp2(fmaxf((rest.m - m) * r.per, kFar)) : 0.f, z = z_rest + z_listed;
  const float inverse = empty ? 0.f : __fdiv_rn(1.f, z), p_rest = z_rest * inverse, p_listed = z_listed * inverse;
  const float t_rest = a.tail && has_rest ? fmaxf(left, 0.f) : 0.f;

  part = 0.f;
  float log_z = 0.f;
  if (a.loss && r.rank == 0) {
    if (r.tid < a.k) {  // the others need no logarithm
      log_z = empty ? 0.f : logf(z);
      for (int j = r.tid; j < a.k; j += kTeam) {
        const float w = t[j] * t_scale;
        if (w > 0.f) part += w * ((l[j] - l_base) - (s[j] - m > -INFINITY ? __fdiv_rn(s[j] - m, temperature) - log_z : -INFINITY));
      }
    }
  }
  // joined behind the gradient, where a barrier is wanted anyway
  const auto write_loss = [&]() {
    float loss = r.team_sum(make_float2(part, 0.f)).x;
    if (r.tid == 0 && r.rank == 0) {
      if (t_rest > 0.f) {
        const float log_p = z_listed <= z_rest ? -log1pf(__fdiv_rn(z_listed, z_rest)) : __fdiv_rn(rest.m - m, temperature) + logf(rest.s) - log_z;
        loss += t_rest * (logf(t_rest) - log_p);
      }
      a.loss[row] = isnan(t_sum) ? NAN : loss;
    }
  };
  if (!a.dscores) return write_loss();

  const float dl = (a.dloss ? a.dloss[row] : a.dloss_all) * (heat ? fminf(__fdiv_rn(1.f, temperature), 3e38f) : 1.f);
  const float coef = has_rest ? dl * __fdiv_rn(t_sum * p_rest - t_rest * p_listed, rest.s) : 0.f * t_sum;
  const float m_rest = has_rest ? rest.m : 0.f;
  const typename R::Out o = r.out(a, row);
  r.asks = false;
  r.put(o, Slope{m_rest, r.per, coef});
  if (a.loss) write_loss();
  if (!a.loss || kTeam == 32) r.team_sync();
  const float mass = t_sum + t_rest;
  for (int j = r.tid; j < a.k; j += kTeam) {
    if (!mine(j)) continue;
    float own = t[j];
    if (twice)
      for (int i = j + 1; i < a.k; i++)
        if (at[i] == at[j]) own += t[i];
    const bool on = s[j] > -INFINITY;
    store_scalar(o.p, o.dtype, at[j] - r.lo, dl * (on ? mass * (weight(j, m) * inverse) - own * t_scale : 0.f * mass));
  }
}

template <typename T>
emr_status distill(Args a, int sms, cudaStream_t st) {
  static std::once_flag once;
  static int fit[kMaxCluster + 1];
  std::call_once(once, [&] { clusters_at_once(distill_kernel<float, 512>, 512, fit); });
  int cluster;
  const int team = plan(a, a.k <= List<32>::kMost ? 32 : 64, sizeof(T), sms, fit, &cluster);
  return team == 32    ? launch_rows(distill_kernel<T, 32>, a, team, cluster, st)
         : team == 64  ? launch_rows(distill_kernel<T, 64>, a, team, cluster, st)
         : team == 128 ? launch_rows(distill_kernel<T, 128>, a, team, cluster, st)
         : team == 256 ? launch_rows(distill_kernel<T, 256>, a, team, cluster, st)
                       : launch_rows(distill_kernel<T, 512>, a, team, cluster, st);
}

}  // namespace

extern "C" emr_status emr_distill(const void* scores, int32_t dtype, int32_t rows, int64_t n, int64_t row_stride, const int32_t* index,
                                  const void* teacher, int32_t teacher_dtype, int32_t k, const float* temperature, float temperature_all,
                                  int32_t tail, const float* dloss, float dloss_all, float* loss, void* dscores, int32_t d_dtype,
                                  int64_t d_stride, void* stream) {
  const emr_status ok = check_scores(scores, dtype, rows, n, row_stride);
  if (ok != EMR_OK) return ok;
  if (!index || !teacher || !dtype_ok(teacher_dtype) || k < 1 || !aligned(index, 4) || !aligned(teacher, dtype_bytes(teacher_dtype)) ||
      !aligned(temperature, 4) || !aligned(dloss, 4) || !aligned(loss, 4) || (!loss && !dscores) || (!temperature && !(temperature_all > 0.f)))
    return EMR_ERR_ARG;
  if (dscores && (!dtype_ok(d_dtype) || d_stride < n || !aligned(dscores, dtype_bytes(d_dtype)) ||
                  overlap(scores, (rows - 1) * row_stride + n, dtype_bytes(dtype), dscores, (rows - 1) * d_stride + n, dtype_bytes(d_dtype))))
    return EMR_ERR_ARG;
  if (k > EMR_MAX_TOP) return EMR_ERR_RANGE;
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  Args a{};
  a.scores = scores, a.n = n, a.row_stride = row_stride, a.rows = rows;
  a.temperature = temperature, a.temperature_all = temperature_all;
  a.dscores = dscores, a.d_dtype = dscores ? d_dtype : EMR_F32, a.d_stride = d_stride;
  a.index = index, a.teacher = teacher, a.teacher_dtype = teacher_dtype, a.k = k, a.tail = tail != 0;
  a.dloss = dloss, a.dloss_all = dloss_all, a.loss = loss;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == EMR_F32) return distill<float>(a, sms, st);
  if (dtype == EMR_BF16) return distill<__nv_bfloat16>(a, sms, st);
  return distill<__half>(a, sms, st);
}
