// Loss on pairs of rollouts (the first of a pair to be preferred) and its gradient: from log-probs, or from logits.
//
//   s_r = sum over r's tokens of (ln pi - ln ref),  x_p = beta (s_c - s_j) - margin,  loss = sum_p w_p l(x_p),
//   D_r = dloss / ds_r = beta sum_p w_p l'(x_p) (1[r = c_p] - 1[r = j_p]),  dz_t = g D_r (onehot(y_t) - softmax(z_t))
//
// A gradient row needs both rollouts of its pairs whole, so logits are read twice: once for the rows' statistics, once for the gradient.
// In between stand sums over tokens (by rollout) and over pairs (by rollout), in whatever order a batch brings them.  They are formed
// exactly, in whole numbers, so that order does not matter: a 32-bit float is m 2^(p - 149) with a 24-bit m, and goes into two of nine
// 64-bit limbs that stand for 2^(32 k - 149) (the low 32 bits of m 2^(p mod 32) and what is above), each below 2^32, so that 2^31 of them fit.
//
// Bound by the bytes of the rows, read twice and written once: 8192 x 151936 bf16, an eighth of them padding, 1060 us: 325 for the statistics (6.7 TB/s), 14 for the sums, 717 for
// the gradient (6.5 TB/s).  Small batches by three launches in a row: 512 x 4096 fp32 14.3 us.  Log-probs alone by launches: 2^20 tokens of 4096 rollouts in 8192 pairs 18.2 us,
// 4096 tokens 7.3.
#include "row_scan.h"

namespace aero {

// ---------------------------------------------------------------------------------- exact sums
enum { kPlusInf = 1, kMinusInf = 2, kNan = 4 };
constexpr int kLimbs = 9;
struct ExactSum {
  unsigned long long limb[kLimbs];
  uint32_t flags;   // of what is not finite
  int32_t count;
};
static_assert(sizeof(ExactSum) == 80, "cleared in 16-byte pieces");

__device__ __forceinline__ void exact_add(ExactSum* s, float x) {
  const uint32_t bits = __float_as_uint(x), e = bits >> 23 & 0xff;
  if (e == 0xff) {
    atomicOr(&s->flags, uint32_t(bits & 0x7fffff ? kNan : bits >> 31 ? kMinusInf : kPlusInf));
    return;
  }
  const uint32_t m = (bits & 0x7fffff) | (e ? 0x800000u : 0u), p = e ? e - 1 : 0;
  if (m == 0) return;
  const uint64_t at = uint64_t(m) << (p & 31);
  const uint64_t low = at & 0xffffffffu, high = at >> 32;
  const uint64_t sign = bits >> 31 ? ~uint64_t(0) : 0;
  unsigned long long* limb = s->limb + (p >> 5);
  if (low) atomicAdd(limb, (unsigned long long)((low ^ sign) - sign));
  if (high) atomicAdd(limb + 1, (unsigned long long)((high ^ sign) - sign));
}
// A 64-bit number to 48 bits.  Beyond 32-bit floats, where the sum of a wave's finite tokens may be (log-probs of the type's lowest value, as masks write them), all 53 of
// them: as a whole number of limb 7's units, 2^75, of which 512 tokens' sum is less than 2^62.
__device__ __forceinline__ void exact_add(ExactSum* s, double x) {
  const float hi = float(x);
  if (fabsf(hi) < INFINITY) {
    exact_add(s, hi);
    exact_add(s, float(x - double(hi)));
  } else if (fabs(x) < INFINITY) {
    const int64_t n = int64_t(x * 0x1p-75);
    atomicAdd(s->limb + 7, (unsigned long long)(n & 0xffffffff));
    atomicAdd(s->limb + 8, (unsigned long long)(n >> 32));   // rounded down: the low limb's part is never negative
  } else {
    exact_add(s, hi);
  }
}
__device__ __forceinline__ double exact_value(const ExactSum& s) {
  if (s.flags) {
    if (s.flags == kPlusInf) return INFINITY;
    if (s.flags == kMinusInf) return -INFINITY;
    return __builtin_nan("");
  }
  int64_t l[kLimbs];
#pragma unroll
  for (int k = 0; k < kLimbs; ++k) l[k] = int64_t(s.limb[k]);
#pragma unroll
  for (int k = 0; k + 1 < kLimbs; ++k) {   // digits of 32 bits, the sign in the last
    l[k + 1] += l[k] >> 32;
    l[k] &= 0xffffffff;
  }
  // a negative sum as its magnitude, or its digits would cancel
  const bool negative = l[kLimbs - 1] < 0;
  if (negative) {
#pragma unroll
    for (int k = 0; k < kLimbs; ++k) l[k] = (k + 1 < kLimbs ? int64_t(0xffffffff) : int64_t(-1)) - l[k];
    l[0] += 1;
  }
  double v = double(l[kLimbs - 1]);
#pragma unroll
  for (int k = kLimbs - 2; k >= 0; --k) v = fma(v, 4294967296.0, double(l[k]));
  v = ldexp(v, -149);
  return negative ? -v : v;
}

// ---------------------------------------------------------------------------------- arguments and workspace
struct PairLoss {
  const int32_t *chosen, *rejected;
  const float* weight;
  int32_t P, R;
  int32_t kind, average;
  float beta, smoothing, margin;
  float *loss, *pair_margin, *rollout_ratio, *drollout;
  int32_t* err_flag;
};

// What a row leaves for the steps behind it.
struct RowRecord {
  int32_t rollout;   // AERO_ROW_PADDING, AERO_ROW_UNTOUCHED: takes no part
  float d;           // logprob - ref
  float offset;      // of the row's exponentials, in powers of two
  float inv;         // 1 / their sum
};
static_assert(sizeof(RowRecord) == 16, "one scalar load");

struct PairWorkspace {
  ExactSum *ratio, *slope;   // [R]
  double* part;              // [ceil(P / 64)] of the loss
  float* gradient;           // [R] of a rollout's log-probs, times grad_scale (T > 0)
  RowRecord* rows;           // [T]
};
constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }
static PairWorkspace carve(void* ws, int64_t T, int32_t R, int32_t P, size_t* bytes) {
  char* p = static_cast<char*>(ws);
  PairWorkspace w;
  const size_t sums = up256(size_t(R) * 2 * sizeof(ExactSum)), part = up256((size_t(P) + 63) / 64 * 8);
  const size_t gradient = T > 0 ? up256(size_t(R) * 4) : 0, rows = up256(size_t(T) * sizeof(RowRecord));
  w.ratio = reinterpret_cast<ExactSum*>(p);
  w.slope = w.ratio + R;
  w.part = reinterpret_cast<double*>(p + sums);
  w.gradient = reinterpret_cast<float*>(p + sums + part);
  w.rows = reinterpret_cast<RowRecord*>(p + sums + part + gradient);
  if (bytes) *bytes = sums + part + gradient + rows;
  return w;
}
size_t preference_workspace_bytes(int64_t T, int32_t R, int32_t P, bool rows) {
  if (R < 0 || P < 0) return 0;
  size_t bytes = 0;
  carve(nullptr, rows ? T : 0, R, P, &bytes);
  return bytes + 256;   // never 0
}

// ---------------------------------------------------------------------------------- a pair
// ln(1 + x), 0 <= x <= 1: 2 artanh s with s = x / (2 + x) <= 1/3, to 1e-10 of itself behind s^18 / 19.
__device__ __forceinline__ double log_1_and(double x) {
  const double s = x / (2.0 + x), q = s * s;
  double y = 1.0 / 17;
#pragma unroll
  for (int n = 15; n > 0; n -= 2) y = fma(y, q, 1.0 / n);
  return 2.0 * s * y;
}
struct PairTerm {
  double value, slope;
};
__device__ __forceinline__ PairTerm pair_term(const PairLoss& a, double x) {
  if (a.kind == AERO_PAIR_HINGE) {
    if (x != x) return PairTerm{x, x};
    return x < 1.0 ? PairTerm{1.0 - x, -1.0} : PairTerm{0.0, 0.0};
  }
  if (a.kind == AERO_PAIR_SQUARE) {
    const double u = (x - 0.5) / double(a.beta);
    return PairTerm{u * u, 2.0 * u / double(a.beta)};
  }
  if (x != x) return PairTerm{x, x};
  const double e = double(a.smoothing), away = exp_of(-fmin(fabs(x), 700.0)), low = log_1_and(away);
  double value = (1.0 - e) * (x < 0.0 ? -x + low : low);
  if (e != 0.0) value += e * (x > 0.0 ? x + low : low);
  const double sigma = x > 0.0 ? away / (1.0 + away) : 1.0 / (1.0 + away);   // of -x
  return PairTerm{value, e - sigma};
}

__device__ __forceinline__ double ratio_of(const PairLoss& a, const ExactSum& s) {
  const double v = exact_value(s);
  return a.average && s.count > 1 ? v / double(s.count) : v;
}
// Derivative by a rollout's log ratio, or with `average` by the log-prob of each of its tokens.
__device__ __forceinline__ float slope_of(const PairLoss& a, const ExactSum& slope, int32_t count) {
  const double v = exact_value(slope);
  return float(a.average && count > 1 ? v / double(count) : v);
}

struct Pair {
  int c, j;
  float w;
};
__device__ __forceinline__ Pair pair_at(const PairLoss& a, int p) {
  return p < a.P ? Pair{a.chosen[p], a.rejected[p], a.weight ? a.weight[p] : 1.f / float(a.P)} : Pair{-1, -1, 0.f};
}
// One pair: its share goes to its rollouts' slopes, its term is returned.
__device__ __forceinline__ double pair_step(const PairLoss& a, int p, const Pair& pair, const ExactSum* ratio, ExactSum* slope) {
  const int c = pair.c, j = pair.j;
  const float w = pair.w;
  double term = 0.0, m = 0.0;
  if (c >= 0 && j >= 0 && (c >= a.R || j >= a.R)) {
    if (a.err_flag) atomicOr(a.err_flag, AERO_DERR_BAD_ROLLOUT);
  } else if (c >= 0 && j >= 0 && w != 0.f) {
    m = double(a.beta) * (ratio_of(a, ratio[c]) - ratio_of(a, ratio[j]));
    const PairTerm t = pair_term(a, m - double(a.margin));
    term = double(w) * t.value;
    const float share = float(double(a.beta) * double(w) * t.slope);
    exact_add(&slope[c], share);
    exact_add(&slope[j], -share);
  }
  if (a.pair_margin) a.pair_margin[p] = float(m);
  return term;
}

// ---------------------------------------------------------------------------------- tokens
// Sums of tokens by rollout, a wave at a time over 64 tokens in a row: as long as they are one rollout's (a rollout's tokens usually stand together), lanes
// add up by themselves and the wave at the end; otherwise rollout by rollout for up to four of them and lane by lane for the others.  What the wave has
// added up waits in a lane of its own, so that many such sums go where they belong at once: each one by itself is as many instructions as all of them.
struct TokenSums {
  ExactSum* sums;
  int rollout = -1;   // uniform; -1: nothing held
  double held = 0.0;
  int count = 0;
  int waiting = 0;    // uniform
  int lane_rollout = 0, lane_count = 0;
  double lane_total = 0.0;

  __device__ __forceinline__ explicit TokenSums(ExactSum* s) : sums(s) {}
  __device__ __forceinline__ void to(int r, double d, int n) {
    exact_add(&sums[r], d);
    atomicAdd(&sums[r].count, n);
  }
  __device__ __forceinline__ void put(int r, double total, int n) {   // the same in every lane
    const bool mine = int(threadIdx.x) % kWave == waiting;
    lane_rollout = mine ? r : lane_rollout;
    lane_total = mine ? total : lane_total;
    lane_count = mine ? n : lane_count;
    if (++waiting == kWave) end();
  }
  __device__ __forceinline__ void flush() {
    if (rollout < 0) return;
    put(rollout, wave_sum_d(held), count);
    rollout = -1;
    held = 0.0;
    count = 0;
  }
  __device__ __forceinline__ void end() {
    if (int(threadIdx.x) % kWave < waiting) to(lane_rollout, lane_total, lane_count);
    waiting = 0;
  }
  __device__ __forceinline__ void add(int r, float d) {   // r < 0: no token
    uint64_t left = __ballot(r >= 0);
    if (left == 0) return;
    const int first = __builtin_amdgcn_readlane(r, __builtin_ctzll(left));
    if (__ballot(r == first) == left) {
      if (first != rollout) {
        flush();
        rollout = first;
      }
      held += r >= 0 ? double(d) : 0.0;
      count += __popcll(left);
      return;
    }
    flush();
    for (int turn = 0; turn < 4 && left; ++turn) {
      const int one = __builtin_amdgcn_readlane(r, __builtin_ctzll(left));
      const uint64_t same = __ballot(r == one);
      put(one, wave_sum_d(r == one ? double(d) : 0.0), __popcll(same));
      left &= ~same;
    }
    if (left >> (threadIdx.x % kWave) & 1) to(r, double(d), 1);
  }
};

// The tokens of the call without logits.
struct Tokens {
  const float *logprob, *ref;
  const int32_t* rollout;
  int64_t T;
};
__device__ __forceinline__ void token_at(const Tokens& k, int64_t t, int64_t end, int R, int32_t* err_flag, int& r, float& d) {
  r = -1;
  d = 0.f;
  if (t >= end) return;
  r = k.rollout[t];
  d = k.logprob[t] - (k.ref ? k.ref[t] : 0.f);   // asked for with the index; no use is made of it where that says so
  if (r >= R && err_flag) atomicOr(err_flag, AERO_DERR_BAD_ROLLOUT);
  if (r < 0 || r >= R) {
    r = -1;
    d = 0.f;
  }
}

// The tokens as rows of logits have left them.
__device__ __forceinline__ void row_token(const RowRecord* rows, int64_t t, int64_t end, int& r, float& d) {
  r = t < end ? max(rows[t].rollout, -1) : -1;
  d = t < end ? rows[t].d : 0.f;
}

// 128 tokens to a wave: 2^20 of them 5.4 us (12.6 MB); with 1024 to a wave 22, as the waves are too few to hide their loads, with 512 12.
constexpr int kTokenRounds = 2, kTokenNT = 256;
template <bool ROWS>
__global__ __launch_bounds__(kTokenNT) void k_pair_tokens(Tokens k, PairLoss a, const RowRecord* __restrict__ rows, ExactSum* ratio) {
  const int64_t from = (int64_t(blockIdx.x) * kTokenNT + threadIdx.x / kWave * kWave) * kTokenRounds + threadIdx.x % kWave;
  int r[kTokenRounds];
  float d[kTokenRounds];
#pragma unroll
  for (int u = 0; u < kTokenRounds; ++u) {
    if constexpr (ROWS) row_token(rows, from + u * kWave, k.T, r[u], d[u]);
    else token_at(k, from + u * kWave, k.T, a.R, a.err_flag, r[u], d[u]);
  }
  TokenSums sums(ratio);
#pragma unroll
  for (int u = 0; u < kTokenRounds; ++u) sums.add(r[u], d[u]);
  sums.flush();
  sums.end();
}

// The sums begin at 0 (a workspace holds anything).
__global__ __launch_bounds__(256) void k_pair_clear(u32x4_t* p, int64_t n) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) p[i] = u32x4_t{0u, 0u, 0u, 0u};
}

// A thread for each pair: two log ratios, the pair's term and its share of two slopes.  Latency: 8192 pairs 6.8 us.
__global__ __launch_bounds__(256) void k_pair_terms(PairLoss a, const ExactSum* __restrict__ ratio, ExactSum* slope, double* __restrict__ part) {
  const int p = blockIdx.x * 256 + threadIdx.x;
  const double term = wave_sum_d(p < a.P ? pair_step(a, p, pair_at(a, p), ratio, slope) : 0.0);
  if (threadIdx.x % kWave == 0 && p < a.P) part[p / kWave] = term;
}

// The rollouts' outputs (gradient: NULL where no row asks for it); the first workgroup adds up the loss.
__global__ __launch_bounds__(256) void k_pair_finish(PairLoss a, const ExactSum* __restrict__ ratio, const ExactSum* __restrict__ slope,
                                                     const double* __restrict__ part, float* __restrict__ gradient, float grad_scale) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < a.R) {
    const float d = slope_of(a, slope[r], ratio[r].count);
    if (a.rollout_ratio) a.rollout_ratio[r] = float(ratio_of(a, ratio[r]));
    if (a.drollout) a.drollout[r] = d;
    if (gradient) gradient[r] = d * grad_scale;
  }
  if (blockIdx.x != 0) return;
  __shared__ double s_part[4];
  double sum = 0.0;
  const int n = (a.P + kWave - 1) / kWave;
  for (int k = threadIdx.x; k < n; k += 256) sum += part[k];
  sum = wave_sum_d(sum);
  if (threadIdx.x % kWave == 0) s_part[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) a.loss[0] = float(s_part[0] + s_part[1] + s_part[2] + s_part[3]);
}

// The pairs by one workgroup, the rollouts' sums in LDS: for as few pairs and rollouts as take it less time than two launches; and the sums over the tokens as
// well where those are few enough (kFromTokens, kFromRows; with kFromSums they are in memory).
enum SumSource { kFromTokens, kFromRows, kFromSums };
constexpr int kSmallNT = 1024, kSmallR = 256, kSmallP = 4096;
template <int SOURCE>
__global__ __launch_bounds__(kSmallNT) void k_pair_small(Tokens k, PairLoss a, const RowRecord* __restrict__ rows, const ExactSum* __restrict__ ratio,
                                                         float* __restrict__ gradient, float grad_scale) {
  constexpr int kAhead = 4;
  __shared__ ExactSum s_ratio[kSmallR], s_slope[kSmallR];
  __shared__ double s_part[kSmallNT / kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  // each wave takes tokens that stand together, in as many rounds as it takes
  const int64_t rounds = (k.T + kSmallNT - 1) / kSmallNT, from = wave * rounds * kWave + lane, end = min(k.T, (wave + 1) * rounds * kWave);
  int r[kAhead];   // the next rounds' tokens, on their way
  float d[kAhead];
  const auto load = [&](int64_t round, int& r, float& d) {
    const int64_t t = from + round * kWave;
    if constexpr (SOURCE == kFromRows) row_token(rows, t, end, r, d);
    else token_at(k, t, end, a.R, a.err_flag, r, d);
  };
  if constexpr (SOURCE != kFromSums) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(u, r[u], d[u]);
  }
  const Pair first_pair = pair_at(a, tid);   // on its way with the tokens
  {
    u32x4_t *p = reinterpret_cast<u32x4_t*>(s_ratio), *q = reinterpret_cast<u32x4_t*>(s_slope);
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(ratio);
    const u32x4_t zero = {0u, 0u, 0u, 0u};
    const int n = a.R * int(sizeof(ExactSum) / 16);
    for (int i = tid; i < n; i += kSmallNT) {
      p[i] = SOURCE == kFromSums ? from[i] : zero;
      q[i] = zero;
    }
  }
  __syncthreads();
  if constexpr (SOURCE != kFromSums) {
    TokenSums sums(s_ratio);
#pragma clang loop unroll(disable)
    for (int64_t round = 0; round < rounds; ++round) {
      const int r_now = r[0];
      const float d_now = d[0];
#pragma unroll
      for (int u = 0; u + 1 < kAhead; ++u) {
        r[u] = r[u + 1];
        d[u] = d[u + 1];
      }
      load(round + kAhead, r[kAhead - 1], d[kAhead - 1]);
      sums.add(r_now, d_now);
    }
    sums.flush();
    sums.end();
    __syncthreads();
  }
  double sum = 0.0;
  if (tid < a.P) sum = pair_step(a, tid, first_pair, s_ratio, s_slope);
  for (int p = tid + kSmallNT; p < a.P; p += kSmallNT) sum += pair_step(a, p, pair_at(a, p), s_ratio, s_slope);
  sum = wave_sum_d(sum);
  if (lane == 0) s_part[wave] = sum;
  __syncthreads();
  for (int i = tid; i < a.R; i += kSmallNT) {
    const float slope = slope_of(a, s_slope[i], s_ratio[i].count);
    if (a.rollout_ratio) a.rollout_ratio[i] = float(ratio_of(a, s_ratio[i]));
    if (a.drollout) a.drollout[i] = slope;
    if (gradient) gradient[i] = slope * grad_scale;
  }
  if (wave == kSmallNT / kWave - 1) {
    const double total = wave_sum_d(lane < kSmallNT / kWave ? s_part[lane] : 0.0);
    if (lane == 0) a.loss[0] = float(total);
  }
}

static bool is_small(int32_t R, int32_t P) { return R <= kSmallR && P <= kSmallP; }
static unsigned blocks_of(int64_t n, int nt) { return unsigned((n + nt - 1) / nt); }

static dim3 token_blocks(int64_t T) { return dim3(blocks_of(T, kTokenNT * kTokenRounds)); }
// Everything behind the sums over the tokens.
static void launch_pairs(const PairLoss& a, const PairWorkspace& w, float* gradient, float grad_scale, hipStream_t s) {
  if (is_small(a.R, a.P)) {
    hipLaunchKernelGGL(k_pair_small<kFromSums>, dim3(1), dim3(kSmallNT), 0, s, Tokens{}, a, nullptr, w.ratio, gradient, grad_scale);
    return;
  }
  if (a.P > 0) hipLaunchKernelGGL(k_pair_terms, dim3(blocks_of(a.P, 256)), dim3(256), 0, s, a, w.ratio, w.slope, w.part);
  hipLaunchKernelGGL(k_pair_finish, dim3(blocks_of(a.R > 1 ? a.R : 1, 256)), dim3(256), 0, s, a, w.ratio, w.slope, w.part, gradient, grad_scale);
}
static void launch_clear(const PairWorkspace& w, int32_t R, hipStream_t s) {
  const int64_t n = int64_t(R) * 2 * int64_t(sizeof(ExactSum)) / 16;
  if (n > 0) hipLaunchKernelGGL(k_pair_clear, dim3(blocks_of(n, 256)), dim3(256), 0, s, reinterpret_cast<u32x4_t*>(w.ratio), n);
}

// ---------------------------------------------------------------------------------- rows of logits
struct PairRows {
  const void* logits;
  int64_t T;
  int V;
  int64_t ld;
  const int32_t* targets;
  const float* ref;
  const int32_t* rollout;
  int R;
  RowRecord* rows;
  int64_t keep_from;    // rows from here on are read by loads that leave them in the caches
  float* logprob_out;
  int32_t* err_flag;
};

// A row's sum of exponentials.  Hundreds of tokens of a rollout add up what their log-probs are off, so what goes the same way in every row counts: summed as elsewhere in this
// library a log-prob of 151936 bf16 logits is 3.9e-7 too high on the average, and a log ratio of 5 over 256 tokens 2.9e-5 of itself.  Three things set it right:
//   - a vector's exponentials are added up before they meet the thread's sum: beside a sampled token that has half of the row, most of them are by themselves less than half a unit of
//     that sum, which stays where it is (1.5e-7 left);
//   - log2 e in 32 bits, l, is off by a relative -1.3e-8, and the row's log-partition by that times the mean logit, which the exponentials times their arguments know (3e-9 left);
//   - an argument is rounded at its own size: the offset follows the largest logit closely, so that the arguments that count are near 0 (not the mean, but what a single log-prob is
//     off: 1.0e-7 -> 0.7e-7, fp32 logits 1.2e-7 -> 0.4e-7).
// Together 0-1 % of the call's time.
//
// With arguments a_j = z_j l - o, S = sum of 2^a_j and m = (sum of 2^a_j a_j) / S:
//   ln pi(y) = a_y ln 2 - ln S + c (a_y - m),  c = (log2 e - l) ln 2 / l,
// to the first order in c times the spread of the logits that count.  All of it is near the offset: what holds for logits around 0 holds for those at 1e9.  (c times the logits
// themselves is not small there, and has to stay out of S, by which the gradient divides exponentials that are formed with l.)
struct RowSum {
  SoftSum st;
  float sa;   // the exponentials times their arguments
};
struct RowTotal {
  SoftTotal st;
  double sa;
};
constexpr float kRowAbove = 2.f;
constexpr float kGone = -256.f;   // an argument whose exponential is 0
constexpr double kLog2eOff = 9.2533473613469254e-9;   // c
template <int N> __device__ __forceinline__ void row_update(RowSum& r, const float (&z)[N]) {
  const float vm = vec_max<N>(z);
  const bool grow = fmaf(vm, kLog2e, -r.st.o) > kRowAbove;
  if (__builtin_amdgcn_ballot_w64(grow) != 0) {
    asm volatile("" ::: "memory");   // stays a branch
    if (grow) {
      const float o = soft_offset(vm), f = exp2_fast(r.st.o - o);
      r.sa = fmaf(r.st.o - o, r.st.s, r.sa) * f;
      r.st = SoftSum{o, r.st.s * f};
    }
  }
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float a = fmaf(z[k], kLog2e, -r.st.o), e = exp2_fast(a);
    s += e;
    r.sa = fmaf(e, fmaxf(a, kGone), r.sa);   // 0 times a masked logit's -inf would be NaN
  }
  r.st.s += s;
}
template <bool WAVE> __device__ __forceinline__ RowTotal row_reduce(const RowTotal& r) {
  const auto most = [](float x, float y) { return fmaxf(x, y); };
  const auto all = [](double x) { return WAVE ? wave_sum_d(x) : row16_sum_d(x); };
  const float o = WAVE ? wave_reduce(r.st.o, most) : row16_reduce(r.st.o, most);
  const double f = double(exp2_fast(r.st.o - o));
  return RowTotal{SoftTotal{o, all(r.st.s * f)}, all(fma(double(r.st.o - o), r.st.s, r.sa) * f)};
}
// Over the workgroup, with the sums of the threads added up in 64 bits.
template <int NT> __device__ __forceinline__ RowTotal row_total(const RowSum& r, RowTotal* lds) {
  RowTotal a = row_reduce<true>(RowTotal{soft_total(r.st), double(r.sa)});
  constexpr int kWaves = NT / kWave;
  if constexpr (kWaves > 1) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (lane == 0) lds[wave] = a;
    __syncthreads();
    a = row_reduce<false>(lane % 16 < kWaves ? lds[lane % 16] : RowTotal{soft_total(soft_identity()), 0.0});
  }
  return a;
}
// The log-prob of a logit; 0 in a row without an unmasked one, NaN in one with a NaN or too large one.
__device__ __forceinline__ double row_logprob(const RowTotal& r, float z) {
  if (r.st.s == 0.0) return 0.0;
  if (r.st.s != r.st.s) return __builtin_nan("");
  if (z <= kMasked) return -INFINITY;
  const double a = fma(double(z), double(kLog2e), -double(r.st.o));   // to 2^-53 of itself
  return fma(a, 0.69314718055994531, kLog2eOff * (a - r.sa / r.st.s)) - log_of(r.st.s);
}

// A thread's part of a row.  KEEP: by loads that leave it in the memory-side cache.
template <int NT, int DT, bool VEC, bool KEEP> __device__ __forceinline__ RowSum row_sum(const RowView<DT, VEC>& row) {
  constexpr int E = RowView<DT, VEC>::E, kAhead = 4;
  const auto load = [&](int i) { return KEEP ? row.load_again(i) : row.load(i); };
  const int tid = threadIdx.x, jr = row.ragged();
  const float zr = jr >= 0 ? row.at(jr) : 0.f;
  RowSum st{soft_identity(), 0.f};
  int i = tid;
  for (; i + (kAhead - 1) * NT < row.nvec; i += kAhead * NT) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = load(i + u * NT);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float z[E];
      row.unpack(v[u], z);
      row_update<E>(st, z);
    }
  }
  for (; i < row.nvec; i += NT) {
    float z[E];
    row.unpack(load(i), z);
    row_update<E>(st, z);
  }
  if (jr >= 0) {
    float z[1] = {zr};
    row_update<1>(st, z);
  }
  return st;
}

// A row's sum of exponentials and its sampled token's log-prob: one workgroup reads it once.  6.7 TB/s from some thousand rows of 151936 bf16 on, 5.2-5.7 for a thousand, which are all under
// way at once and end together.  256 and 1024 threads instead of 512: 0-3 % longer; eight vectors ahead 0-1 %.
template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_pair_rows(PairRows a) {
  __shared__ RowTotal lds[NT / kWave];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const int r = a.rollout[t], y = a.targets[t];
  if (r < 0 || y < 0 || r >= a.R || y >= a.V) {   // uniform
    if (tid == 0) {
      if (r >= 0 && y >= 0 && a.err_flag) atomicOr(a.err_flag, r >= a.R ? AERO_DERR_BAD_ROLLOUT : AERO_DERR_BAD_TARGET);
      a.rows[t] = RowRecord{r == AERO_ROW_UNTOUCHED ? AERO_ROW_UNTOUCHED : AERO_ROW_PADDING, 0.f, 0.f, 0.f};
      if (a.logprob_out) a.logprob_out[t] = 0.f;
    }
    return;
  }
  const RowView<DT, VEC> row(a.logits, t, a.ld, a.V);
  const float zy = row.at(y);
  const RowSum st = t < a.keep_from ? row_sum<NT, DT, VEC, false>(row) : row_sum<NT, DT, VEC, true>(row);
  const RowTotal sum = row_total<NT>(st, lds);
  if (tid != 0) return;
  const bool empty = sum.st.s == 0.0;
  const double lp = row_logprob(sum, zy);
  const float d = empty ? 0.f : float(a.ref ? lp - double(a.ref[t]) : lp);
  a.rows[t] = RowRecord{empty ? AERO_ROW_PADDING : r, d, sum.st.o, float(1.0 / sum.st.s)};
  if (a.logprob_out) a.logprob_out[t] = float(lp);
}

// ---------------------------------------------------------------------------------- gradient rows
// dz_j = k exp2(z_j log2 e - offset) + g 1[j = y], k = -g / sum of the exponentials.
struct RowGradient {
  float g, k, offset;
  int y;
  template <int DT> __device__ __forceinline__ float at(float z, int j) const {
    const float d = k * exp2_fast(fmaf(z, kLog2e, -offset));
    return j == y ? d + g : d;
  }
};

// (row, segment) per workgroup, a vector per thread, in the order of addresses from the end: what was read last is read first.  Stored past the caches, which
// hold the rows then: 1000 rows of 151936 bf16 88 -> 80 us (7.2 TB/s, a part of it not from memory), 8192 rows 755 -> 717.  A vector asked for before it is known that its
// rollout has a gradient takes 0.1-0.8 % less, but a satisfied hinge leaves most rows unread.
template <int NT, int DT>
__global__ __launch_bounds__(NT) void k_pair_grad_seg(const void* logits, int V, int64_t ld, int segs, const RowRecord* __restrict__ rows,
                                                      const float* __restrict__ gradient, const int32_t* __restrict__ targets, void* dlogits) {
  constexpr int E = Storage<DT>::kPerVec;
  const unsigned block = gridDim.x - 1 - blockIdx.x;
  const int64_t t = block / segs;
  const int seg = block % segs;
  const RowRecord row = rows[t];
  if (row.rollout == AERO_ROW_UNTOUCHED) return;
  const RowGeom geom = row_geom<DT>(logits, t, ld, V);
  const char* zrow = row_ptr<DT>(logits, t, ld);
  char* drow = row_ptr<DT>(dlogits, t, ld);
  const u32x4_t* zv = reinterpret_cast<const u32x4_t*>(zrow + geom.head * Storage<DT>::kBytes);
  u32x4_t* dv = reinterpret_cast<u32x4_t*>(drow + geom.head * Storage<DT>::kBytes);
  const int k = seg * NT + threadIdx.x;
  const bool in = k < geom.nvec;
  const int jr = seg == 0 ? ragged_elt<DT>(geom, V, threadIdx.x) : -1;
  const float g = row.rollout >= 0 ? gradient[row.rollout] : 0.f;
  if (g == 0.f) {   // uniform: nothing to read
    if (in) __builtin_nontemporal_store(u32x4_t{0u, 0u, 0u, 0u}, dv + k);
    if (jr >= 0) store_elt<DT>(drow, jr, 0.f);
    return;
  }
  u32x4_t v = {0u, 0u, 0u, 0u};
  if (in) v = zv[k];
  const RowGradient c{g, -g * row.inv, row.offset, targets[t]};
  if (in) {
    float z[E], d[E];
    unpack_vec<DT>(v, z);
#pragma unroll
    for (int e = 0; e < E; ++e) d[e] = c.k * exp2_fast(fmaf(z[e], kLog2e, -c.offset));
    const int at = c.y - geom.head;
    if (k == (at >> Storage<DT>::kLogPerVec)) {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] += e == (at & (E - 1)) ? c.g : 0.f;
    }
    __builtin_nontemporal_store(pack_vec<DT>(d), dv + k);
  }
  if (jr >= 0) store_elt<DT>(drow, jr, c.at<DT>(load_elt<DT>(zrow, jr), jr));
}

// A row per workgroup, element by element: where logits and dlogits differ in their offset from 16 bytes, or a launch would not
// hold the segments.
template <int DT>
__global__ __launch_bounds__(256) void k_pair_grad_row(const void* logits, int V, int64_t ld, const RowRecord* __restrict__ rows,
                                                       const float* __restrict__ gradient, const int32_t* __restrict__ targets, void* dlogits) {
  const int64_t t = blockIdx.x;
  const RowRecord row = rows[t];
  if (row.rollout == AERO_ROW_UNTOUCHED) return;
  const float g = row.rollout >= 0 ? gradient[row.rollout] : 0.f;
  const RowGradient c{g, -g * row.inv, row.offset, targets[t]};
  const char* zrow = row_ptr<DT>(logits, t, ld);
  char* drow = row_ptr<DT>(dlogits, t, ld);
  for (int j = threadIdx.x; j < V; j += 256) store_elt<DT>(drow, j, g == 0.f ? 0.f : c.at<DT>(load_elt<DT>(zrow, j), j));
}

template <int DT> static void launch_rows(const PairRows& a, hipStream_t s) {
  const bool vec = rows_alike(a.logits, nullptr, Storage<DT>::kBytes);
  const int64_t work = vec ? (a.V + Storage<DT>::kPerVec - 1) / Storage<DT>::kPerVec : a.V;
  const dim3 grid = dim3(unsigned(a.T));
  auto launch = [&](auto nt) {
    if (vec) hipLaunchKernelGGL((k_pair_rows<nt.value, DT, true>), grid, dim3(nt.value), 0, s, a);
    else hipLaunchKernelGGL((k_pair_rows<nt.value, DT, false>), grid, dim3(nt.value), 0, s, a);
  };
  if (work <= 4 * 64) launch(std::integral_constant<int, 64>{});
  else if (work <= 16 * 256) launch(std::integral_constant<int, 256>{});
  else if (a.T <= compute_units()) launch(std::integral_constant<int, 1024>{});
  else launch(std::integral_constant<int, 512>{});
}

template <int DT> static void launch_grad(const PairRows& a, const float* gradient, void* dlogits, hipStream_t s) {
  const int64_t nvec = a.V / Storage<DT>::kPerVec + 1;
  const int nt = nvec <= 128 ? 64 : 256;
  const int64_t segs = (nvec + nt - 1) / nt;
  if (!rows_alike(a.logits, dlogits, Storage<DT>::kBytes) || !grid_fits(a.T * segs, nt)) {
    hipLaunchKernelGGL(k_pair_grad_row<DT>, dim3(unsigned(a.T)), dim3(256), 0, s, a.logits, a.V, a.ld, a.rows, gradient, a.targets, dlogits);
    return;
  }
  const auto kernel = nt == 64 ? k_pair_grad_seg<64, DT> : k_pair_grad_seg<256, DT>;
  hipLaunchKernelGGL(kernel, dim3(unsigned(a.T * segs)), dim3(nt), 0, s, a.logits, a.V, a.ld, int(segs), a.rows, gradient, a.targets, dlogits);
}

// The memory-side cache holds 256 MB: that much of the rows' end is still there when the gradient, which goes through the rows from their end, reads it.  Rows of
// 300 MB 140 us (1000 x 151936 bf16) with nothing kept, 133 with this, 140 with all of them; 2.5 GB 1067 / 1060 / 1078.
constexpr int64_t kKeptBytes = int64_t(256) << 20;

// Up to so many tokens one workgroup also adds them up, which saves a clearing launch and one for the sums.  One launch / three, us, of 16 and 256 rollouts: 512 tokens
// 6.2 / 10.2, 6.9 / 11.1; 4096 7.3 / 10.2, 11.8 / 11.6; 8192 8.6 / 10.3, 14.3 / 11.3; 16384 10.7 / 10.5, 19.0 / 11.0; as rows of 512 logits 512 13.1 / 16.7, 14.0 / 17.8;
// 4096 16.8 / 17.9, 21.1 / 20.3; 8192 21.6 / 21.1, 27.3 / 23.5.
constexpr int64_t kOneRows = 4096, kOneTokens = 8192;

template <int DT> static void run_rows(const PairRows& rows, const PairLoss& a, const PairWorkspace& w, float grad_scale, void* dlogits, hipStream_t s) {
  const bool small = rows.T <= kOneRows && is_small(a.R, a.P);
  if (!small) launch_clear(w, a.R, s);
  PairRows r = rows;
  r.keep_from = dlogits ? r.T - kKeptBytes / (int64_t(r.V) * Storage<DT>::kBytes) : r.T;
  if (r.T > 0) launch_rows<DT>(r, s);
  const Tokens k{nullptr, nullptr, nullptr, r.T};
  float* gradient = dlogits && r.T > 0 ? w.gradient : nullptr;   // read by the rows alone; without any the workspace has no room for it
  if (small) {
    hipLaunchKernelGGL(k_pair_small<kFromRows>, dim3(1), dim3(kSmallNT), 0, s, k, a, r.rows, nullptr, gradient, grad_scale);
  } else {
    if (r.T > 0) hipLaunchKernelGGL(k_pair_tokens<true>, token_blocks(r.T), dim3(kTokenNT), 0, s, k, a, r.rows, w.ratio);
    launch_pairs(a, w, gradient, grad_scale, s);
  }
  if (gradient) launch_grad<DT>(r, gradient, dlogits, s);
}

// ---------------------------------------------------------------------------------- the calls' checks
static bool finite(float x) { return x - x == 0.f; }
static aero_status check_pairs(const aero_preference_params* p, int32_t R, int32_t P, const int32_t* chosen, const int32_t* rejected,
                               const float* loss) {
  if (!p || !loss) return AERO_ERR_NULL;
  if (R < 0 || P < 0 || R >= (1 << 22) || P >= (1 << 22)) return AERO_ERR_SHAPE;
  if (p->kind != AERO_PAIR_LOGISTIC && p->kind != AERO_PAIR_HINGE && p->kind != AERO_PAIR_SQUARE) return AERO_ERR_SHAPE;
  if ((p->average != 0 && p->average != 1) || !(p->beta > 0.f) || !finite(p->beta) || !finite(p->margin)) return AERO_ERR_SHAPE;
  if (p->kind == AERO_PAIR_LOGISTIC && !(p->smoothing >= 0.f && p->smoothing <= 0.5f)) return AERO_ERR_SHAPE;
  if (P > 0 && (!chosen || !rejected)) return AERO_ERR_NULL;
  return AERO_OK;
}
static bool workspace_ok(const void* ws, size_t bytes, size_t need) { return ws && reinterpret_cast<uintptr_t>(ws) % 256 == 0 && bytes >= need; }

}  // namespace aero

extern "C" aero_status aero_preference_loss(
    const float* logprob, int64_t T, const float* ref_logprob, const int32_t* token_rollout, int32_t R, const int32_t* pair_chosen,
    const int32_t* pair_rejected, const float* pair_weight, int32_t P, const aero_preference_params* params, float* loss, float* pair_margin,
    float* rollout_ratio, float* drollout, int32_t* err_flag, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (T < 0 || T >= (int64_t(1) << 25)) return AERO_ERR_SHAPE;
  const aero_status st = check_pairs(params, R, P, pair_chosen, pair_rejected, loss);
  if (st != AERO_OK) return st;
  if (T > 0 && (!logprob || !token_rollout)) return AERO_ERR_NULL;
  if (!workspace_ok(workspace, workspace_bytes, preference_workspace_bytes(T, R, P, false))) return AERO_ERR_WORKSPACE;
  const PairWorkspace w = carve(workspace, 0, R, P, nullptr);
  const PairLoss a{pair_chosen, pair_rejected, pair_weight, P, R, params->kind, params->average, params->beta, params->smoothing, params->margin,
                   loss, pair_margin, rollout_ratio, drollout, err_flag};
  const Tokens k{logprob, ref_logprob, token_rollout, T};
  hipStream_t s = as_stream(stream);
  if (T <= kOneTokens && is_small(R, P)) {
    hipLaunchKernelGGL(k_pair_small<kFromTokens>, dim3(1), dim3(kSmallNT), 0, s, k, a, nullptr, nullptr, nullptr, 0.f);
    return launch_status();
  }
  launch_clear(w, R, s);
  if (T > 0) hipLaunchKernelGGL(k_pair_tokens<false>, token_blocks(T), dim3(kTokenNT), 0, s, k, a, nullptr, w.ratio);
  launch_pairs(a, w, nullptr, 0.f, s);
  return launch_status();
}

extern "C" aero_status aero_preference_loss_bwd(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld, const int32_t* targets, const float* ref_logprob,
    const int32_t* token_rollout, int32_t R, const int32_t* pair_chosen, const int32_t* pair_rejected, const float* pair_weight, int32_t P,
    const aero_preference_params* params, float grad_scale, float* loss, float* pair_margin, float* rollout_ratio, float* logprob_out,
    void* dlogits, int32_t* err_flag, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (T < 0 || T >= (1 << 22) || V < 1 || V > (1 << 24) || ld < V) return AERO_ERR_SHAPE;
  if (!storage_dtype_ok(dtype)) return AERO_ERR_DTYPE;
  const aero_status st = check_pairs(params, R, P, pair_chosen, pair_rejected, loss);
  if (st != AERO_OK) return st;
  if (T > 0 && (!logits || !targets || !token_rollout)) return AERO_ERR_NULL;
  if (!workspace_ok(workspace, workspace_bytes, preference_workspace_bytes(T, R, P, true))) return AERO_ERR_WORKSPACE;
  const PairWorkspace w = carve(workspace, T, R, P, nullptr);
  const PairLoss a{pair_chosen, pair_rejected, pair_weight, P, R, params->kind, params->average, params->beta, params->smoothing, params->margin,
                   loss, pair_margin, rollout_ratio, nullptr, err_flag};
  const PairRows rows{logits, T, V, ld, targets, ref_logprob, token_rollout, R, w.rows, 0, logprob_out, err_flag};
  hipStream_t s = as_stream(stream);
  switch (dtype) {
    case AERO_BF16: run_rows<kBF16>(rows, a, w, grad_scale, dlogits, s); break;
    case AERO_F16: run_rows<kF16>(rows, a, w, grad_scale, dlogits, s); break;
    case AERO_F8E4M3: run_rows<kF8>(rows, a, w, grad_scale, dlogits, s); break;
    default: run_rows<kF32>(rows, a, w, grad_scale, dlogits, s);
  }
  return launch_status();
}
