// Verification of drafted tokens against the policy's rows, from given random numbers.
//
// The first launch forms the running sums of every row that can matter (target rows up to the count of drafted tokens,
// the draft rows in front of it), a row split over several workgroups; with many sequences it also decides position by position, so that
// rows behind a refusal are mostly left out.  The second finds the first position whose uniform number is not below p / q, and in every
// slice of the vocabulary the largest max(0, p - q) / noise there.  The third joins a sequence's slices: the larger score, the lower id
// where equal, which does not depend on their order.  (Joining in the second launch by its last workgroup, with the slices' keys as plain
// stores, takes a device-wide fence per workgroup, 50 of 129 us for 128 sequences; keys that are atomics themselves have not been measured.)  Short rows take one launch, in which a workgroup does all of that for a sequence.
//
// Bound by the rows' and the noise's bytes (151936 bf16: 128 sequences of up to 5 drafted tokens 71 us, of which the sums 41 at 5.6 TB/s and
// the draw 28; 256 of 3 copied tokens 86 us) and, for few sequences, by three launches (8 of 4 tokens 16.9 us).  The noise is the
// caller's: a [B, V] fp32 row a sequence, 31 and 44 % of the bytes of those two.
#include <algorithm>

#include "row_scan.h"

namespace aero {

constexpr int kVerifyParts = 8, kMaxSlices = 64;   // most parts of a row in the first launch, slices of a draw in the second

struct VerifyArgs {
  const void *target, *draft;
  int B, G, V;
  int64_t ld;
  const int32_t *tokens, *count;
  const float *uniform, *noise;
  int32_t* accepted;
  int32_t* out;
  float* logprob;
  int32_t* err_flag;
  SoftSum* sums;      // [B * (2 G + 1)][parts]: target rows, then draft rows
  uint64_t* best;     // [B][slices]: largest score and its id
  double* lse;        // [B]: of the row that is drawn from
  int32_t* refused;   // [B]: first position known to be refused
  double* lp;         // [B * (G + 1)]: ln p of a drafted token that was accepted, NaN of one that was refused
  int parts, slices;
};

// Drafted tokens of a sequence that count: up to its count, and to the first id outside the vocabulary.  -1: idle.  Every lane of the
// wave gets it; token = this lane's drafted id.
__device__ __forceinline__ int drafted(const VerifyArgs& a, int b, int lane, int& token, int32_t& flags) {
  const int n = a.count ? a.count[b] : a.G;
  token = lane < a.G ? a.tokens[int64_t(b) * a.G + lane] : -1;
  flags = 0;
  if (n < 0 || n > a.G) {
    if (n > a.G) flags = AERO_DERR_BAD_COUNT;
    return -1;
  }
  const uint64_t bad = __builtin_amdgcn_ballot_w64(lane < n && (token < 0 || token >= a.V));
  if (!bad) return n;
  const int first = __builtin_ctzll(bad);
  if (__builtin_amdgcn_readlane(token, first) >= a.V) flags = AERO_DERR_BAD_TARGET;
  return first;
}

template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_verify_rows(VerifyArgs a) {
  constexpr int E = RowView<DT, VEC>::E, kAhead = VEC ? 4 : 8;
  __shared__ SoftSum s_sum[NT / kWave];
  const int tid = threadIdx.x, part = blockIdx.y, parts = gridDim.y;
  const int64_t r = blockIdx.x, n_target = int64_t(a.B) * (a.G + 1);
  const bool is_target = r < n_target;
  const int width = is_target ? a.G + 1 : a.G;
  const int64_t rr = is_target ? r : r - n_target;
  const int b = int(rr / width), i = int(rr % width);
  int token;
  int32_t flags;
  const int n = drafted(a, b, tid % kWave, token, flags);
  if (is_target ? i > n : i >= n) return;   // uniform
  const RowView<DT, VEC> row(is_target ? a.target : a.draft, rr, a.ld, a.V);
  const int per = (row.nvec + parts - 1) / parts;
  const int first = min(part * per, row.nvec), last = min(first + per, row.nvec);
  const int jr = part == 0 ? row.ragged() : -1;
  SoftSum st = soft_identity();
  if (jr >= 0) {
    float z[1] = {row.at(jr)};
    soft_update<1>(st, z);
  }
  int k = first + tid;
  for (; k + (kAhead - 1) * NT < last; k += kAhead * NT) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = row.load(k + u * NT);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float z[E];
      row.unpack(v[u], z);
      soft_update<E>(st, z);
    }
  }
  for (; k < last; k += NT) {
    float z[E];
    row.unpack(row.load(k), z);
    soft_update<E>(st, z);
  }
  st = soft_block_reduce<NT>(st, s_sum);
  if (tid == 0) a.sums[r * parts + part] = st;
}

// The parts of a row's sum, all asked for at once, and the row's sum from them.
struct RowParts {
  SoftSum part[kVerifyParts];
  __device__ __forceinline__ void load(const VerifyArgs& a, int64_t r) {
#pragma unroll
    for (int p = 0; p < kVerifyParts; ++p) part[p] = p < a.parts ? a.sums[r * a.parts + p] : soft_identity();
  }
  __device__ __forceinline__ SoftSum sum() const {
    SoftSum st = part[0];
#pragma unroll
    for (int p = 1; p < kVerifyParts; ++p) st = soft_merge(st, part[p]);
    return st;
  }
};
__device__ __forceinline__ SoftSum from_lane(SoftSum s, int lane) {
  return SoftSum{__int_as_float(__builtin_amdgcn_readlane(__float_as_int(s.o), lane)),
                 __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s.s), lane))};
}

// Is a drafted token accepted, u q < p (has_q: q is the softmax of a row, else 1), from its logits and its rows' sums?  lp: its ln p.  Masks are looked
// at first: the differences of masked logits, or of one and an empty row's -inf, say nothing about the probabilities, which are 0.
__device__ __forceinline__ bool accept(float u, float zp, SoftSum p, bool has_q, float zq, SoftSum q, double& lp) {
  const double lse_p = soft_lse(p);
  lp = double(zp) - lse_p;
  if (!(zp > kMasked) || !(lse_p - lse_p == 0.0)) return false;   // p = 0, or the row is empty or has a NaN
  double ratio = lp;
  if (has_q) {   // uniform
    const double lse_q = soft_lse(q);
    if (!(lse_q - lse_q == 0.0)) return false;
    if (!(zq > kMasked)) return true;   // u 0 < p
    ratio -= double(zq) - lse_q;
  }
  // beyond +-800 the ratio is past every number that u may be: a number of 0 is below any ratio, any other above e^-800
  return u == 0.f || double(u) < exp_of(fmin(fmax(ratio, -800.0), 800.0));
}

// Many sequences: a workgroup per position, which goes over its target row and its draft row together and decides.  Positions
// are the slow index of the grid, so that those behind a refused one, whose rows nobody needs, mostly find it refused when their turn comes; where they do
// not, they are worked on for nothing.
__global__ void k_verify_start(int32_t* refused, int B) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b < B) refused[b] = INT32_MAX;
}
template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_verify_positions(VerifyArgs a) {
  using View = RowView<DT, VEC>;
  constexpr int E = View::E, kAhead = 2;
  __shared__ SoftSum s_sum[2][NT / kWave];
  const int tid = threadIdx.x, i = blockIdx.x / a.B, b = blockIdx.x % a.B;
  if (__hip_atomic_load(a.refused + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < i) return;   // uniform; an old value only costs time
  int token;
  int32_t flags;
  const int n = drafted(a, b, tid % kWave, token, flags);
  if (i > n) return;   // uniform
  const int x = i < n ? __builtin_amdgcn_readlane(token, i) : 0;
  const bool minus = a.draft && i < n;
  const int64_t rt = int64_t(b) * (a.G + 1) + i, rd = int64_t(b) * a.G + min(i, a.G - 1), n_target = int64_t(a.B) * (a.G + 1);
  const View prow(a.target, rt, a.ld, a.V), qrow(minus ? a.draft : a.target, minus ? rd : rt, a.ld, a.V);
  const float zp = prow.at(x), zq = qrow.at(x), u = i < n ? a.uniform[rd] : 0.f;
  SoftSum p = soft_identity(), q = soft_identity();
  auto ragged = [&](const View& row, SoftSum& st) {
    const int jr = row.ragged();
    if (jr >= 0) {
      float z[1] = {row.at(jr)};
      soft_update<1>(st, z);
    }
  };
  auto fold = [&](const u32x4_t& v, SoftSum& st) {
    float z[E];
    View::unpack(v, z);
    soft_update<E>(st, z);
  };
  ragged(prow, p);
  if (minus) ragged(qrow, q);
  const int nvec = minus ? min(prow.nvec, qrow.nvec) : prow.nvec;   // the rows' vectors differ by one at most
  int k = tid;
  for (; k + (kAhead - 1) * NT < nvec; k += kAhead * NT) {
    u32x4_t v[kAhead], w[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = prow.load(k + j * NT);
    if (minus) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) w[j] = qrow.load(k + j * NT);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) fold(v[j], p);
    if (minus) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) fold(w[j], q);
    }
  }
  for (; k < prow.nvec || (minus && k < qrow.nvec); k += NT) {
    if (k < prow.nvec) fold(prow.load(k), p);
    if (minus && k < qrow.nvec) fold(qrow.load(k), q);
  }
  p = soft_block_reduce<NT>(p, s_sum[0]);
  if (minus) q = soft_block_reduce<NT>(q, s_sum[1]);
  if (tid == 0) {
    a.sums[rt] = p;
    if (minus) a.sums[n_target + rd] = q;
    if (i < n) {
      double lp;
      const bool ok = accept(u, zp, p, minus, zq, q, lp);
      a.lp[rt] = ok ? lp : __builtin_nan("");
      if (!ok) atomicMin(a.refused + b, i);
    }
  }
}

// Largest score so far and its column.
struct Drawn {
  float score;
  int j;
};
__device__ __forceinline__ void race(Drawn& d, float score, int j) {
  if (score > d.score) d = Drawn{score, j};   // columns ascend within a thread
}
// (score, lowest id) as a number that grows with the score; 0: none.
__device__ __forceinline__ uint64_t drawn_key(Drawn d) {
  return d.score > 0.f ? (uint64_t(__float_as_uint(d.score)) << 32) | uint32_t(~d.j) : 0;
}
// The largest over the workgroup, in its first thread; one barrier.
template <int NT> __device__ __forceinline__ uint64_t block_drawn(Drawn d, uint64_t* lds /*[NT/64]*/) {
  const int lane = threadIdx.x % kWave;
  const float most = wave_reduce(d.score, [](float x, float y) { return fmaxf(x, y); });
  d.j = -wave_max_i(d.score == most ? -d.j : INT32_MIN + 1);
  d.score = most;
  if (lane == 0) lds[threadIdx.x / kWave] = drawn_key(d);
  __syncthreads();
  uint64_t key = 0;
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) key = lds[w] > key ? lds[w] : key;
  }
  return key;
}

// E elements from column j on, or floats, at any element's alignment.
template <int DT, bool VEC> __device__ __forceinline__ u32x4_t load_elts(const char* row, int j) {
  if constexpr (VEC) return *reinterpret_cast<const u32x4_any_t*>(row + int64_t(j) * Storage<DT>::kBytes);
  else return u32x4_t{__float_as_uint(load_elt<DT>(row, j)), 0u, 0u, 0u};
}
template <int E> __device__ __forceinline__ void load_floats(const float* x, float (&y)[E]) {
  if constexpr (E == 1) {
    y[0] = x[0];
  } else {
#pragma unroll
    for (int k = 0; k < E; k += 4) {
      const f32x4_any_t v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any_t*>(x + k));
      y[k] = v.x; y[k + 1] = v.y; y[k + 2] = v.z; y[k + 3] = v.w;
    }
  }
}
// The sequence's drawn token from its best key, which the first thread has.  Where the residual vanishes (rows that are the same but for
// roundings) it is drawn from p, by this workgroup alone; so it does where what is left is a masked logit's exponential, which beside logits next to
// AERO_LOGIT_LIMIT may be 2^-120 for 0.
template <int NT, int DT>
__device__ __forceinline__ void put_drawn(const VerifyArgs& a, int b, int n, double lse, uint64_t key, uint64_t* lds /*[NT/64]*/) {
  __shared__ uint64_t s_best;
  const int64_t rt = int64_t(b) * (a.G + 1) + n;
  const char* const row = row_ptr<DT>(a.target, rt, a.ld);
  float z = 0.f;
  const auto look = [&]() {   // the first thread's token's logit; no key where it is masked
    z = key ? load_elt<DT>(row, int(~uint32_t(key))) : 0.f;
    if (z <= kMasked) key = 0;
  };
  if (threadIdx.x == 0) {
    look();
    s_best = key;
  }
  __syncthreads();
  if (s_best == 0 && lse - lse == 0.0) {   // uniform
    Drawn d{0.f, 0};
    for (int j = threadIdx.x; j < a.V; j += NT) {
      const float y = load_elt<DT>(row, j);
      if (y > kMasked) race(d, expf(float(double(y) - lse)) * __builtin_amdgcn_rcpf(a.noise[int64_t(b) * a.V + j]), j);
    }
    key = block_drawn<NT>(d, lds);   // the barrier above lies between two uses of lds
    if (threadIdx.x == 0) look();
  }
  if (threadIdx.x == 0) {
    a.out[rt] = key ? int(~uint32_t(key)) : -1;
    if (a.logprob) a.logprob[rt] = key ? float(double(z) - lse) : 0.f;
  }
}

// The sum of a row by a wave.
template <int DT, bool VEC> __device__ __forceinline__ SoftSum wave_row(const RowView<DT, VEC>& row) {
  constexpr int E = RowView<DT, VEC>::E, kAhead = 4;
  const int lane = threadIdx.x % kWave;
  SoftSum st = soft_identity();
  auto fold = [&](const u32x4_t& v) {
    float z[E];
    row.unpack(v, z);
    soft_update<E>(st, z);
  };
  const int jr = VEC ? ragged_elt<DT>(RowGeom{row.head, row.nvec}, row.V, lane) : -1;
  if (jr >= 0) {
    float z[1] = {row.at(jr)};
    soft_update<1>(st, z);
  }
  int k = lane;
  for (; k + (kAhead - 1) * kWave < row.nvec; k += kAhead * kWave) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = row.load_again(k + u * kWave);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) fold(v[u]);
  }
  for (; k < row.nvec; k += kWave) fold(row.load_again(k));
  return soft_reduce<true>(st);
}

// What is known before: the rows' sums by k_verify_rows, decisions too by k_verify_positions, or nothing (short rows: a wave forms the sum of a row,
// and one launch does everything).  With one slice the drawn token too, else what k_verify_end needs.
enum { kSummed, kDecided, kAlone };
template <int NT, int DT, bool VEC, int KNOWN>
__global__ __launch_bounds__(NT) void k_verify_draw(VerifyArgs a) {
  constexpr bool DECIDED = KNOWN == kDecided;
  __shared__ SoftSum s_row[KNOWN == kAlone ? 2 * AERO_DRAFT_MAX + 1 : 1];
  constexpr int E = RowView<DT, VEC>::E;
  __shared__ uint64_t s_key[NT / kWave];
  const int tid = threadIdx.x, lane = tid % kWave, b = blockIdx.x, slice = blockIdx.y, slices = gridDim.y;
  // ---- lane i: position i.  Everything that the count does not decide is asked for together with it; what belongs to positions
  // behind it may never have been written and is not used. ----
  const int64_t n_target = int64_t(a.B) * (a.G + 1);
  const int64_t my_t = int64_t(b) * (a.G + 1) + min(lane, a.G), my_d = int64_t(b) * a.G + min(lane, a.G - 1);
  const bool minus = a.draft != nullptr;   // and so G > 0
  RowParts pp, qp;
  if constexpr (KNOWN != kAlone) {
    pp.load(a, my_t);
    if (minus) qp.load(a, n_target + my_d);
  }
  double lp = 0.0;
  float u = 0.f;
  if constexpr (DECIDED) lp = a.lp[my_t];
  else u = lane < a.G ? a.uniform[my_d] : 0.f;
  int token;
  int32_t flags;
  const int count = drafted(a, b, lane, token, flags);
  if (slice == 0 && tid == 0 && flags && a.err_flag) atomicOr(a.err_flag, flags);
  int32_t* const out = a.out + int64_t(b) * (a.G + 1);
  float* const lp_out = a.logprob ? a.logprob + int64_t(b) * (a.G + 1) : nullptr;
  if (count < 0) {   // uniform
    if (slice == 0 && tid <= a.G) {
      if (tid == 0) a.accepted[b] = 0;
      out[tid] = -1;
      if (lp_out) lp_out[tid] = 0.f;
    }
    return;
  }
  const bool on = lane < count;
  SoftSum sp, sq;
  if constexpr (KNOWN == kAlone) {
    const int rows = count + 1 + (minus ? count : 0);   // target rows, then draft rows
    for (int r = tid / kWave; r < rows; r += NT / kWave) {
      const bool of_draft = r > count;
      const RowView<DT, VEC> row(of_draft ? a.draft : a.target, of_draft ? int64_t(b) * a.G + r - count - 1 : int64_t(b) * (a.G + 1) + r, a.ld, a.V);
      const SoftSum st = wave_row(row);
      if (lane == 0) s_row[r] = st;
    }
    __syncthreads();
    sp = lane <= count ? s_row[lane] : soft_identity();
    sq = minus && on ? s_row[count + 1 + lane] : soft_identity();
  } else {
    sp = pp.sum();
    sq = minus ? qp.sum() : soft_identity();
  }
  bool ok;
  if constexpr (DECIDED) {
    ok = on && lp == lp;
  } else {
    const int column = on ? token : 0;
    const float zp = load_elt<DT>(row_ptr<DT>(a.target, my_t, a.ld), column);
    const float zq = minus ? load_elt<DT>(row_ptr<DT>(a.draft, my_d, a.ld), column) : 0.f;
    ok = accept(u, zp, sp, minus, zq, sq, lp) && on;
  }
  const int n = __builtin_ctzll(~__builtin_amdgcn_ballot_w64(ok));   // at most 63 positions
  const bool refused = n < count;
  const int own = refused && !minus ? __builtin_amdgcn_readlane(token, n) : -1;   // the whole of q

  // ---- the draw: this workgroup's slice of row n ----
  const int64_t rt = int64_t(b) * (a.G + 1) + n, rd = int64_t(b) * a.G + n;
  const SoftSum pt = from_lane(sp, n);
  const double lse = soft_lse(pt);
  if (slice == 0 && tid <= a.G) {
    if (tid == 0) {
      a.accepted[b] = n;
      a.lse[b] = lse;
    }
    if (tid != n) {   // the drawn token follows
      out[tid] = tid < n ? token : -1;
      if (lp_out) lp_out[tid] = tid < n ? float(lp) : 0.f;
    }
  }
  Drawn left{0.f, 0};
  if (lse - lse == 0.0) {   // finite
    const SoftSum qt = refused && minus ? from_lane(sq, n) : soft_identity();
    const double lse_q = soft_lse(qt);
    const bool less = lse_q - lse_q == 0.0;
    const float op = -pt.o, ip = 1.f / pt.s, oq = less ? -qt.o : 0.f, iq = less ? 1.f / qt.s : 0.f;
    const RowView<DT, VEC> prow(a.target, rt, a.ld, a.V);
    const char* const qrow = less ? row_ptr<DT>(a.draft, rd, a.ld) : nullptr;
    const float* const noise = a.noise + int64_t(b) * a.V;
    auto consider = [&](float z, float y, float e, int j) {
#pragma clang fp contract(off)   // equal probabilities leave nothing
      const float p = ip * exp2_fast(fmaf(z, kLog2e, op)), q = iq * exp2_fast(fmaf(y, kLog2e, oq));
      race(left, (j == own ? 0.f : p - q) * __builtin_amdgcn_rcpf(e), j);
    };
    const int per = (prow.nvec + slices - 1) / slices;
    const int first = min(slice * per, prow.nvec), last = min(first + per, prow.nvec);
    constexpr int kAhead = VEC ? 2 : 4;
    for (int i0 = first + tid; i0 < last; i0 += kAhead * NT) {
      u32x4_t zv[kAhead], yv[kAhead];
      float e[kAhead][E];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = min(i0 + k * NT, last - 1), j = prow.column(i);
        load_floats<E>(noise + j, e[k]);
        zv[k] = prow.load_again(i);
        yv[k] = u32x4_t{0u, 0u, 0u, 0u};
        if (less) yv[k] = load_elts<DT, VEC>(qrow, j);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i0 + k * NT >= last) break;
        float z[E], y[E];
        prow.unpack(zv[k], z);
        prow.unpack(yv[k], y);
        const int j = prow.column(i0 + k * NT);
#pragma unroll
        for (int c = 0; c < E; ++c) consider(z[c], y[c], e[k][c], j + c);
      }
    }
    const int jr = slice == 0 ? prow.ragged() : -1;
    if (jr >= 0) {   // a tie goes to the lower id, which is not the later one here
      const Drawn before = left;
      left = Drawn{0.f, 0};
      consider(prow.at(jr), less ? load_elt<DT>(qrow, jr) : 0.f, noise[jr], jr);
      left = drawn_key(before) > drawn_key(left) ? before : left;
    }
  }
  const uint64_t key = block_drawn<NT>(left, s_key);
  if (slices == 1) put_drawn<NT, DT>(a, b, n, lse, key, s_key);   // uniform
  else if (tid == 0) a.best[int64_t(b) * slices + slice] = key;
}

// The slices of a sequence into its drawn token.
constexpr int kEndNT = 256;
template <int DT> __global__ __launch_bounds__(kEndNT) void k_verify_end(VerifyArgs a) {
  __shared__ uint64_t s_key[kEndNT / kWave];
  const int tid = threadIdx.x, b = blockIdx.x;
  const int count = a.count ? a.count[b] : a.G;
  if (count < 0 || count > a.G) return;   // uniform
  static_assert(kMaxSlices <= kEndNT, "a slice per thread");
  const uint64_t x = tid < a.slices ? a.best[int64_t(b) * a.slices + tid] : 0;
  const uint64_t key = block_drawn<kEndNT>(x ? Drawn{__uint_as_float(uint32_t(x >> 32)), int(~uint32_t(x))} : Drawn{0.f, 0}, s_key);
  put_drawn<kEndNT, DT>(a, b, a.accepted[b], a.lse[b], key, s_key);
}

// Workgroups that a row's sum is split over: 8 to a CU in all.  (151936 bf16, 72 rows: 2 / 4 / 8 parts 9.9 / 8.3 / 7.6 us; 1408 rows, of which
// 768 are read: 1 / 2 / 4 parts 43.7 / 41.0 / 41.5.)
static int verify_parts(int64_t rows, int nvec, int NT) {
  return int(std::max<int64_t>(1, std::min<int64_t>({kVerifyParts, (8 * compute_units() + rows - 1) / rows, nvec / (2 * NT)})));
}
// Workgroups that the draw of a sequence is split over: one to a CU in all, since each goes through the decision first.  (8 sequences: 4 / 16 /
// 32 / 37 slices 14.2 / 7.8 / 7.4 / 9.4 us; 128: 2 / 8 / 32 slices 27.9 / 29.6 / 41.2.)
static int verify_slices(int64_t B, int nvec, int NT) {
  return int(std::max<int64_t>(1, std::min<int64_t>({kMaxSlices, compute_units() / B, nvec / NT})));
}

struct VerifyWorkspace {
  SoftSum* sums;
  uint64_t* best;
  double* lse;
  double* lp;
  int32_t* refused;
  size_t bytes;
};
static VerifyWorkspace verify_workspace(void* base, int64_t rows, int64_t B) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  char* const p = reinterpret_cast<char*>(base);
  VerifyWorkspace w;
  size_t at = 0;
  auto take = [&](size_t n) {
    char* const q = p + at;
    at += up(n);
    return q;
  };
  w.sums = reinterpret_cast<SoftSum*>(take(size_t(2 * rows) * kVerifyParts * sizeof(SoftSum)));
  w.best = reinterpret_cast<uint64_t*>(take(size_t(B) * kMaxSlices * 8));
  w.lse = reinterpret_cast<double*>(take(size_t(B) * 8));
  w.lp = reinterpret_cast<double*>(take(size_t(rows) * 8));
  w.refused = reinterpret_cast<int32_t*>(take(size_t(B) * 4));
  w.bytes = at + 256;
  return w;
}
size_t verify_workspace_bytes(int64_t rows, int32_t V, int32_t B) {
  (void)V;
  return verify_workspace(nullptr, rows, B > 0 ? B : 0).bytes;
}

// One launch, a workgroup a sequence and a wave a row?  By the vectors that a lane goes through: few enough, or more where the sequences alone fill the CUs.  Two
// or three launches / one, bf16 (vectors): 1 sequence x 3 copied tokens of 1024 (2) 7.0 / 5.7 us, 8 x 4 of 3000 (6) 9.2 / 8.3, of 11000 (22) 13.4 / 14.1, 256 x 3 of
// 1024 16.3 / 7.4, of 16000 (32) 26.6 / 19.6, 1 x 8 of 5586 (22) 9.3 / 11.6.  (Rows split over the waves that have none: 1 us more at 1024, nothing gained below
// 32000.)  Where workgroups queue the bound falls, since all rows are read and by position those behind a refusal mostly are not: 512 x 5 of 16384 (32) 49 / 45, of
// 32000 (63) 82 / 91, 1024 x 5 of 8192 (16) 69 / 56, of 16384 93 / 97, 4096 x 5 of 8192 246 / 228, of 16384 316 / 361, of 32000 513 / 651; and so it does, further, for fewer
// rows than four, which leave most waves idle: nothing drafted, 512 x 4096 (8) 11.4 / 12.1, 1024 x 2048 (4) 14.3 / 19.0, 4096 x 8192 59 / 126; one token with the drafter's
// rows, 512 x 8192 0.85 of the time, 1024 x 8192 37 / 40, 4096 x 4096 99 / 107.
static bool verify_alone(int64_t B, int64_t rows, int nvec) {
  constexpr int kWaves = 1024 / kWave;
  const int64_t each = (rows + kWaves - 1) / kWaves * ((nvec + kWave - 1) / kWave);
  if (B <= 256) return each <= 12 + B / 8;
  if (rows < 4) return each <= (rows == 1 ? 2048 : 10240) / B;
  return each <= (B <= 1024 ? 32 : 20);
}

template <int DT, bool VEC> static void verify_launch(VerifyArgs a, hipStream_t s) {
  constexpr int NT = 512;
  const int64_t positions = int64_t(a.B) * (a.G + 1), rows = positions + (a.draft ? int64_t(a.B) * a.G : 0);
  const int nvec = a.V / RowView<DT, VEC>::E;
  a.slices = verify_slices(a.B, nvec, NT);
  const dim3 draw{unsigned(a.B), unsigned(a.slices)};
  // Otherwise, from four positions to a CU on: rows one by one / by position, 256 sequences x 8 drafted tokens 260 / 192 us, x 3 142 / 134, x 3 copied
  // ones 94.0 / 91.8; fewer: 128 x 5 102 / 100, with drawn counts 75 / 85, 64 x 4 49.9 / 53.4
  if (verify_alone(a.B, rows / a.B, nvec)) {
    a.slices = 1;
    hipLaunchKernelGGL((k_verify_draw<1024, DT, VEC, kAlone>), dim3(unsigned(a.B)), dim3(1024), 0, s, a);
  } else if (a.G > 0 && positions >= 4 * compute_units()) {
    a.parts = 1;
    hipLaunchKernelGGL(k_verify_start, dim3(unsigned((a.B + 255) / 256)), dim3(256), 0, s, a.refused, a.B);
    // 1024 threads, so that two positions are under way on a CU (512, four: 223 / 141 / 97.2 us)
    hipLaunchKernelGGL((k_verify_positions<1024, DT, VEC>), dim3(unsigned(positions)), dim3(1024), 0, s, a);
    hipLaunchKernelGGL((k_verify_draw<NT, DT, VEC, kDecided>), draw, dim3(NT), 0, s, a);
  } else {
    a.parts = verify_parts(rows, nvec, NT);
    hipLaunchKernelGGL((k_verify_rows<NT, DT, VEC>), dim3(unsigned(rows), unsigned(a.parts)), dim3(NT), 0, s, a);
    hipLaunchKernelGGL((k_verify_draw<NT, DT, VEC, kSummed>), draw, dim3(NT), 0, s, a);
  }
  if (a.slices > 1) hipLaunchKernelGGL((k_verify_end<DT>), dim3(unsigned(a.B)), dim3(kEndNT), 0, s, a);
}

}  // namespace aero

extern "C" aero_status aero_verify_draft(const void* target_logits, const void* draft_logits, int32_t dtype, int32_t B, int32_t G,
                                         int32_t V, int64_t ld, const int32_t* draft_tokens, const int32_t* draft_count,
                                         const float* uniform, const float* noise, int32_t* accepted, int32_t* tokens, float* logprob,
                                         int32_t* err_flag, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (B < 0 || G < 0 || V < 1 || V > (1 << 24) || ld < V) return AERO_ERR_SHAPE;
  if (G > AERO_DRAFT_MAX) return AERO_ERR_LIMIT;
  if (!grid_fits(int64_t(B) * (2 * G + 1), 1024)) return AERO_ERR_SHAPE;
  if (!storage_dtype_ok(dtype)) return AERO_ERR_DTYPE;
  if (B == 0) return AERO_OK;
  if (!target_logits || !noise || !accepted || !tokens || (G > 0 && (!draft_tokens || !uniform))) return AERO_ERR_NULL;
  const int64_t rows = int64_t(B) * (G + 1);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < verify_workspace_bytes(rows, V, B))
    return AERO_ERR_WORKSPACE;
  const VerifyWorkspace ws = verify_workspace(workspace, rows, B);
  const VerifyArgs a{target_logits, G > 0 ? draft_logits : nullptr, B, G, V, ld, draft_tokens, draft_count, uniform, noise, accepted, tokens,
                     logprob, err_flag, ws.sums, ws.best, ws.lse, ws.refused, ws.lp, 1, 1};
  const bool vec = rows_alike(target_logits, nullptr, storage_bytes(dtype)) && rows_alike(a.draft, nullptr, storage_bytes(dtype));
  const hipStream_t s = as_stream(stream);
  switch (dtype) {
    case AERO_BF16: vec ? verify_launch<kBF16, true>(a, s) : verify_launch<kBF16, false>(a, s); break;
    case AERO_F16: vec ? verify_launch<kF16, true>(a, s) : verify_launch<kF16, false>(a, s); break;
    case AERO_F8E4M3: vec ? verify_launch<kF8, true>(a, s) : verify_launch<kF8, false>(a, s); break;
    default: vec ? verify_launch<kF32, true>(a, s) : verify_launch<kF32, false>(a, s);
  }
  return launch_status();
}
