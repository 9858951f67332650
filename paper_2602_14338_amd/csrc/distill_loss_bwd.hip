// Distillation from a teacher's top logits: divergence of each row from its list, and the gradient row.
//
// With q = softmax(z), the list's ids i_k with probabilities p_k and everything else as one event of probability p_r:
//   L = sum_k p_k (ln p_k - ln q(i_k)) + p_r (ln p_r - ln q_r),   P = sum p + p_r,
//   dL/dz_j = P q_j - p_j (listed),  (P - p_r / q_r) q_j (others);
// the renormalised form is p_k / sum p with p_r = 0.  So a gradient row is one multiple of the exponentials, replaced at
// the K listed places.
//
// q_r is what a converging drafter makes small, and 1 - sum q(i_k) would leave nothing of it: the sum over the row leaves the
// listed places out (they count as masked while it runs) and their K exponentials are added to it.  Each thread knows from a
// chain of the entries that fall into its vectors which of them hold listed places, so that all other vectors pay one
// comparison; in the gradient row the listed places are stored over what the others' multiple left there.
//
// Bound by the bytes of a row, read once and written once: 8192 x 32000 fp16 held in registers 183 us (5.4 TB/s), 8192 x 151936 bf16 streaming through
// registers and LDS 875-890 us (5.3 TB/s; an elementwise copy of the same rows 1040); small batches by a row's chain and the launch of the loss
// sum: 2048 x 1024 fp32 7.7 + 1.8 us.
#include <algorithm>
#include <mutex>

#include "row_scan.h"

namespace aero {

constexpr int kListMax = AERO_TOPK_MAX;
constexpr int kListWaves = kListMax / kWave;

struct DistillArgs {
  const void* logits;
  int64_t T;
  int V;
  int64_t ld;
  const int32_t* index;
  const float* logprob;
  int K;
  const float* weight;
  int tail;
  float grad_scale;
  float *term, *row_loss;
  void* dlogits;
  int32_t* err_flag;
};

// The entries of a row's list by the thread that looks after their place (thread = vector % NT).  A place within a thread is the number
// of its vector there times E plus the element; kRagged: the thread's element outside the vectors.
constexpr int kRagged = 0xffff;
template <int NT> struct ListPlaces {
  int32_t head[NT];         // first entry of a thread's chain, -1: none
  int16_t next[kListMax];
  uint16_t place[kListMax];
  float p[kListMax], z[kListMax];   // teacher probability, logit
};

// One entry as its thread holds it, and what a wave of them adds up to.
struct ListEntry {
  int j;      // id, -1: absent
  double p, lp;
  float z;
};
struct ListSums {
  double mass, p_lp_z;   // sum p, sum p (ln p - z)
  SoftTotal own;         // of the listed logits
  int32_t any, bad;      // entries; ids outside the vocabulary, or the same place twice
};

// The list's ids find their threads.  entry.j >= V has been told apart before.
template <int NT, int DT, bool VEC>
__device__ __forceinline__ void list_place(ListPlaces<NT>& list, const RowView<DT, VEC>& row, int k, int j) {
  constexpr int E = RowView<DT, VEC>::E;
  const int at = j - row.head;
  int owner, place;
  if (at >= 0 && at < row.nvec * E) {
    owner = at / E % NT;
    place = at / E / NT * E + at % E;
  } else {
    owner = at < 0 ? j : E + at - row.nvec * E;
    place = kRagged;
  }
  list.place[k] = uint16_t(place);
  list.next[k] = int16_t(atomicExch(&list.head[owner], k));
}
// After the barrier behind list_place: is the entry's place taken by another entry further down the chain?
template <int NT> __device__ __forceinline__ bool list_twice(const ListPlaces<NT>& list, int k) {
  bool twice = false;
  for (int e = list.next[k]; e >= 0; e = list.next[e]) twice |= list.place[e] == list.place[k];
  return twice;
}
// Calls f(entry, place) for this thread's entries.
template <int NT, class F> __device__ __forceinline__ void each_listed(const ListPlaces<NT>& list, F f) {
  for (int k = list.head[threadIdx.x]; k >= 0; k = list.next[k]) f(k, int(list.place[k]));
}
// This thread's listed places as bits, for N vectors of E elements, and whether its ragged element is one.
template <int N, int E> struct PlaceBits {
  static constexpr int kWords = (N * E + 31) / 32;
  uint32_t bits[kWords];
  bool ragged;
  template <int NT> __device__ __forceinline__ explicit PlaceBits(const ListPlaces<NT>& list) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) bits[i] = 0;
    ragged = false;
    each_listed(list, [&](int, int place) {
      ragged |= place == kRagged;
      const uint32_t bit = 1u << (place % 32);
#pragma unroll
      for (int i = 0; i < kWords; ++i) bits[i] |= place / 32 == i ? bit : 0;
    });
  }
  // the listed logits of vector u count as masked
  __device__ __forceinline__ void mask(float (&z)[E], int u) const {
    static_assert(32 % E == 0, "a vector's bits are in one word");
    const uint32_t word = bits[u * E / 32];
    const int shift = u * E % 32;
    if (word >> shift & ((1u << E) - 1)) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t m = uint32_t(__builtin_amdgcn_sbfe(int(word), shift + e, 1));   // all ones or zeros
        z[e] = __uint_as_float((m & 0xff800000u) | (~m & __float_as_uint(z[e])));      // -inf or the logit
      }
    }
  }
};

// Probability of a listed log-prob, in 64 bits: a loss is a small difference, and what p_k rounds by is what it is off by.  0 where 32 bits hold
// no probability.
__device__ __forceinline__ double list_prob(float lp) {
  const double p = exp_of(double(lp));
  return lp < -103.97f ? 0.0 : p;
}

// Sums over the entries of a wave, left in s[wave] by its first lane.
__device__ __forceinline__ void list_sum(const ListEntry& e, bool bad, ListSums* s) {
  ListSums sum;
  const bool there = e.j >= 0;
  SoftSum own = soft_identity();
  if (there && !(e.z <= kMasked)) {
    float z[1] = {e.z};
    soft_update<1>(own, z);
  }
  sum.own = soft_reduce<true>(soft_total(own));
  sum.mass = wave_sum_d(there ? e.p : 0.0);
  sum.p_lp_z = wave_sum_d(there && e.p != 0.0 ? e.p * (e.lp - (e.z <= kMasked ? -INFINITY : double(e.z))) : 0.0);
  sum.any = __builtin_amdgcn_ballot_w64(there) != 0;
  sum.bad = __builtin_amdgcn_ballot_w64(bad) != 0;
  if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = sum;
}

__device__ __forceinline__ void put_loss(const DistillArgs& a, int64_t t, float w, float loss) {
  a.term[t] = loss == 0.f ? 0.f : w * loss;   // a quiet row's weight may be anything
  if (a.row_loss) a.row_loss[t] = loss;
}
// The same value in every lane, said to the compiler: it lives in a scalar register.
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// A gradient vector: at_other 2^(z log2 e - o_rest), and at the listed places at_listed 2^(z log2 e - o_all) - scale_p p.  The others'
// coefficient is taken relative to their own softmax, (P - p_r / q_r) q_j = (P q_r - p_r) q_j / q_r, so that it stays bounded however
// little mass they have.
struct RowGrad {
  float at_other, o_rest, at_listed, o_all, scale_p;
  bool quiet;   // no loss, no gradient
};
// What the sum over the other places and the list come to; one thread writes the loss (a quiet row's too).  By all threads.
__device__ __forceinline__ RowGrad row_terms(const DistillArgs& a, int64_t t, float w, SoftTotal rest, const ListSums* s, int waves, bool bad = false,
                                              bool report = true) {
  double mass = 0.0, p_lp_z = 0.0;
  SoftTotal all = rest;
  bool any = false;
  for (int k = 0; k < waves; ++k) {   // uniform
    mass += s[k].mass;
    p_lp_z += s[k].p_lp_z;
    all = soft_merge(all, s[k].own);
    any |= s[k].any != 0;
    bad |= s[k].bad != 0;
  }
  const bool has_rest = rest.s != 0.0, renorm = a.tail == AERO_TAIL_RENORM;
  // the difference of the offsets first: far from 0 a sum may be 2^64 and more, or 2^-64, for a logit (see kMasked)
  const float rest_q = has_rest ? float(rest.s) * exp2_fast(rest.o - all.o) / float(all.s) : 0.f;
  const double g = double(w) * double(a.grad_scale);
  const double rest_p = renorm || !has_rest || mass >= 1.0 ? 0.0 : 1.0 - mass;
  const double total = renorm ? 1.0 : mass + rest_p;
  RowGrad r;
  r.quiet = bad || !any || all.s == 0.0 || (renorm && mass == 0.0);
  r.scale_p = uniform(float(renorm ? g / mass : g));
  r.at_listed = uniform(float(g * total) / float(all.s));
  r.o_all = uniform(all.o);
  r.at_other = uniform(has_rest ? float(g * (total * double(rest_q) - rest_p)) / float(rest.s) : 0.f);
  r.o_rest = uniform(rest.o);
  if (report && threadIdx.x == blockDim.x - 1) {   // the first wave has the list to look after
    if (bad && a.err_flag) atomicOr(a.err_flag, AERO_DERR_BAD_TEACHER);
    double loss = 0.0;
    if (!r.quiet) {
      const double lse = soft_lse(all);
      if (renorm) {
        loss = p_lp_z / mass - log_of(mass) + lse;
      } else {
        loss = p_lp_z + (mass != 0.0 ? mass * lse : 0.0);
        if (rest_p != 0.0) loss += rest_p * (log_of(rest_p) - (soft_lse(rest) - lse));
      }
    }
    put_loss(a, t, w, float(loss));
  }
  return r;
}

// A vector of the gradient row as if none of its places were listed, and the listed ones over it: the thread that stored a vector
// stores them behind it, so that they land in that order.
template <int E> __device__ __forceinline__ void grad_elts(const float (&z)[E], float (&d)[E], const RowGrad& r) {
#pragma unroll
  for (int e = 0; e < E; ++e) d[e] = r.at_other * exp2_fast(fmaf(z[e], kLog2e, -r.o_rest));
}
template <int NT, int DT, bool VEC>
__device__ __forceinline__ void put_listed(const ListPlaces<NT>& list, const RowView<DT, VEC>& row, const RowGrad& r, char* drow, int jr,
                                           int from = 0, int to = kRagged) {   // places, of which the ragged one is its thread's with jr >= 0
  constexpr int E = RowView<DT, VEC>::E;
  each_listed(list, [&](int k, int place) {
    if (place == kRagged ? jr < 0 : place < from || place >= to) return;
    const int j = place == kRagged ? jr : row.head + (place / E * NT + int(threadIdx.x)) * E + place % E;
    store_elt<DT>(drow, j, r.at_listed * exp2_fast(fmaf(list.z[k], kLog2e, -r.o_all)) - r.scale_p * list.p[k]);
  });
}

// Any row, read twice: by one workgroup (kWhole), or split over gridDim.y workgroups that find the sums in one launch (kSums) and write
// the gradient in a second (kGradient).  A part is whole turns of the workgroup's threads.
enum { kWhole, kSums, kGradient };
constexpr int kMaxParts = 16;
struct RowSplit {
  SoftTotal part[kMaxParts];
  ListSums list;
};
template <int STEP, int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_distill_row(DistillArgs a, int summed, RowSplit* __restrict__ splits) {   // summed: parts of the sums
  using View = RowView<DT, VEC>;
  constexpr int E = View::E, kAhead = 4, kWaves = NT / kWave;
  static_assert(NT >= kListMax, "an entry per thread");
  __shared__ ListPlaces<NT> list;
  __shared__ SoftTotal s_sum[kWaves];
  __shared__ ListSums s_list[kListWaves];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, K = a.K, part = blockIdx.y, parts = gridDim.y;
  const float w = a.weight[t];
  const View row(a.logits, t, a.ld, a.V);
  const int turns = (row.nvec + NT - 1) / NT, per = (turns + parts - 1) / parts;
  const int first = min(part * per, turns), nvec = min(min(first + per, turns) * NT, row.nvec);   // of this part
  const int jr = part == 0 ? row.ragged() : -1;
  char* const drow = a.dlogits ? row_ptr<DT>(a.dlogits, t, a.ld) : nullptr;
  RowSplit* const split = STEP == kWhole ? nullptr : splits + t;
  auto put = [&](int vec, const float (&d)[E]) {
    if constexpr (VEC)
      __builtin_nontemporal_store(pack_vec<DT>(d), reinterpret_cast<u32x4_t*>(drow + row.head * Storage<DT>::kBytes) + vec);
    else
      store_elt<DT>(drow, vec, d[0]);
  };
  auto zero_fill = [&]() {
    if (STEP == kSums || !drow) return;
    float zero[E];
#pragma unroll
    for (int e = 0; e < E; ++e) zero[e] = 0.f;
    for (int i = first * NT + tid; i < nvec; i += NT) put(i, zero);
    if (jr >= 0) store_elt<DT>(drow, jr, 0.f);
  };
  if (w == 0.f) {   // uniform
    if (STEP != kSums && part == 0 && tid == 0) put_loss(a, t, w, 0.f);
    zero_fill();
    return;
  }
  list.head[tid] = -1;
  __syncthreads();
  ListEntry entry{-1, 0.0, 0.0, 0.f};
  bool bad = false;
  if (tid < K) {
    entry.j = a.index[t * K + tid];
    bad = entry.j >= a.V;
    if (bad) entry.j = -1;
    if (entry.j >= 0) {
      const float lp = a.logprob[t * K + tid];
      entry.lp = double(lp);
      entry.z = row.at(entry.j);
      list_place(list, row, tid, entry.j);
      entry.p = list_prob(lp);
      list.p[tid] = float(entry.p);
      list.z[tid] = entry.z;
    }
  }
  __syncthreads();
  const float zr = jr >= 0 ? row.at(jr) : 0.f;
  SoftSum st = soft_identity();
  SoftTotal total = soft_total(st);
  if constexpr (STEP != kGradient) {
    if (tid < kListMax) {   // whole waves
      if (entry.j >= 0) bad |= list_twice(list, tid);
      list_sum(entry, bad, s_list);
    }
    const bool chained = list.head[tid] >= 0;
    auto fold = [&](const u32x4_t& v, int turn) {
      float z[E];
      View::unpack(v, z);
      if (chained)
        each_listed(list, [&](int, int place) {
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] = place == turn * E + e ? -INFINITY : z[e];
        });
      soft_update<E>(st, z);
    };
    int turn = first, i = first * NT + tid;
    for (; i + (kAhead - 1) * NT < nvec; i += kAhead * NT, turn += kAhead) {
      u32x4_t v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = row.load_again(i + u * NT);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) fold(v[u], turn + u);
    }
    for (; i < nvec; i += NT) fold(row.load_again(i), turn++);
    if (jr >= 0) {
      float z[1] = {zr};
      each_listed(list, [&](int, int place) { z[0] = place == kRagged ? -INFINITY : z[0]; });
      soft_update<1>(st, z);
    }
    total = soft_block_total<NT>(st, s_sum);   // its barrier: s_list
  }
  if constexpr (STEP == kSums) {
    if (tid == 0) {
      split->part[part] = total;
      if (part == 0) {
        ListSums all = s_list[0];
#pragma unroll
        for (int k = 1; k < kListWaves; ++k) {
          all.mass += s_list[k].mass;
          all.p_lp_z += s_list[k].p_lp_z;
          all.own = soft_merge(all.own, s_list[k].own);
          all.any |= s_list[k].any;
          all.bad |= s_list[k].bad;
        }
        split->list = all;
      }
    }
    return;
  }
  if constexpr (STEP == kGradient) {
    if (tid % 16 < summed) total = split->part[tid % 16];
    total = soft_reduce<false>(total);
  }
  const RowGrad r = row_terms(a, t, w, total, STEP == kGradient ? &split->list : s_list, STEP == kGradient ? 1 : kListWaves, false, part == 0);
  if (!drow) return;
  if (r.quiet) {   // uniform
    zero_fill();
    return;
  }

  auto turned = [&](const u32x4_t& v, int vec) {
    float z[E], d[E];
    View::unpack(v, z);
    grad_elts<E>(z, d, r);
    put(vec, d);
  };
  int i = first * NT + tid;
  for (; i + (kAhead - 1) * NT < nvec; i += kAhead * NT) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = row.load(i + u * NT);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) turned(v[u], i + u * NT);
  }
  for (; i < nvec; i += NT) turned(row.load(i), i);
  if (jr >= 0) store_elt<DT>(drow, jr, r.at_other * exp2_fast(fmaf(zr, kLog2e, -r.o_rest)));
  put_listed(list, row, r, drow, jr, first * E, (first + per) * E);
}

// One workgroup per row, which its threads hold: kHeldVecs vectors each in registers.
constexpr int kHeldVecs = 8;
template <int NT, int DT>
__global__ __launch_bounds__(NT) void k_distill_held(DistillArgs a) {
  using View = RowView<DT, true>;
  constexpr int E = View::E, kWaves = NT / kWave;
  __shared__ ListPlaces<NT> list;
  __shared__ SoftTotal s_sum[kWaves];
  __shared__ ListSums s_list[kListWaves];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, K = a.K;
  const float w = a.weight[t];
  int j = -1;
  float lp = 0.f;
  if (tid < K) {   // asked for ahead of what depends on the weight
    j = a.index[t * K + tid];
    lp = a.logprob[t * K + tid];
  }
  const View row(a.logits, t, a.ld, a.V);
  const int nvec = row.nvec, jr = row.ragged();
  char* const drow = a.dlogits ? row_ptr<DT>(a.dlogits, t, a.ld) : nullptr;
  const __amdgpu_buffer_rsrc_t src = row.buffer(row.row), dst = row.buffer(drow ? drow : row.row);
  const uint32_t voff = uint32_t(tid) * 16u;
  auto zero_fill = [&]() {
    if (!drow) return;
    const u32x4_t zero = {0u, 0u, 0u, 0u};
    for (int i = tid; i < nvec; i += NT) __builtin_amdgcn_raw_buffer_store_b128(zero, dst, uint32_t(i) * 16u, 0, 2);
    if (jr >= 0) store_elt<DT>(drow, jr, 0.f);
  };
  if (w == 0.f) {   // uniform
    if (tid == 0) put_loss(a, t, w, 0.f);
    zero_fill();
    return;
  }
  ListEntry entry{j, 0.0, 0.0, 0.f};
  bool bad = j >= a.V;
  if (bad) entry.j = -1;
  if (entry.j >= 0) entry.z = row.at(entry.j);
  u32x4_t v[kHeldVecs];
#pragma unroll
  for (int u = 0; u < kHeldVecs; ++u) v[u] = __builtin_amdgcn_raw_buffer_load_b128(src, voff + uint32_t(u) * (NT * 16u), 0, 2);
  const float zr = jr >= 0 ? row.at(jr) : 0.f;
  list.head[tid] = -1;
  __syncthreads();
  if (entry.j >= 0) {
    entry.lp = double(lp);
    list_place(list, row, tid, entry.j);
    entry.p = list_prob(lp);
    list.p[tid] = float(entry.p);
    list.z[tid] = entry.z;
  }
  __syncthreads();
  const int list_waves = (K + kWave - 1) / kWave;
  if (tid < list_waves * kWave) {
    if (entry.j >= 0) bad |= list_twice(list, tid);
    list_sum(entry, bad, s_list);
  }
  const PlaceBits<kHeldVecs, E> listed(list);
  SoftSum st = soft_identity();
#pragma unroll
  for (int u = 0; u < kHeldVecs; ++u) {
    if (tid < nvec - u * NT) {
      float z[E];
      View::unpack(v[u], z);
      listed.mask(z, u);
      soft_update<E>(st, z);
    }
    __builtin_amdgcn_sched_barrier(0);   // one vector at a time: keeps temporaries from piling up
  }
  if (jr >= 0) {
    float z[1] = {listed.ragged ? -INFINITY : zr};
    soft_update<1>(st, z);
  }
  // orders the loads of the row before the stores over it, for a gradient in place: by its barrier, and with one wave because
  // every lane's result needs every lane's loads
  const SoftTotal rest = soft_block_total<NT>(st, s_sum);
  if constexpr (kWaves == 1) __syncthreads();
  const RowGrad r = row_terms(a, t, w, rest, s_list, list_waves);
  if (!drow) return;
  if (r.quiet) {   // uniform
    zero_fill();
    return;
  }
  uint32_t voff_st = voff;
  asm volatile("" : "+v"(voff_st));   // the store offsets are formed again; the load offsets need not stay
#pragma unroll
  for (int u = 0; u < kHeldVecs; ++u) {
    if (tid < nvec - u * NT) {
      float z[E], d[E];
      View::unpack(v[u], z);
      grad_elts<E>(z, d, r);
      __builtin_amdgcn_raw_buffer_store_b128(pack_vec<DT>(d), dst, voff_st + uint32_t(u) * (NT * 16u), 0, 2);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (jr >= 0) store_elt<DT>(drow, jr, r.at_other * exp2_fast(fmaf(zr, kLog2e, -r.o_rest)));
  put_listed(list, row, r, drow, jr);
}

// The rows with a weight in front, then the others, each in no particular order.  ctr[0], ctr[1]: rows placed from the front and from
// the back.  ONE: a single workgroup, which counts in LDS and needs no launch in front of it.
constexpr int kOrderNT = 1024;
__global__ void k_distill_start(int32_t* ctr) { ctr[threadIdx.x] = 0; }
template <bool ONE>
__global__ __launch_bounds__(kOrderNT) void k_distill_order(int64_t T, const float* __restrict__ weight, int32_t* __restrict__ ctr,
                                                            int32_t* __restrict__ order) {
  __shared__ int32_t own[2];
  const int lane = threadIdx.x % kWave;
  if constexpr (ONE) {
    if (threadIdx.x < 2) own[threadIdx.x] = 0;
    __syncthreads();
  }
  int32_t* const count = ONE ? own : ctr;
  for (int64_t t0 = int64_t(blockIdx.x) * kOrderNT; t0 < T; t0 += int64_t(gridDim.x) * kOrderNT) {   // uniform
    const int64_t t = t0 + threadIdx.x;
    const bool in = t < T, need = in && weight[t] != 0.f;
    const uint64_t m_need = __builtin_amdgcn_ballot_w64(need), m_rest = __builtin_amdgcn_ballot_w64(in && !need);
    const uint64_t below = (uint64_t(1) << lane) - 1;
    int front = 0, back = 0;
    if (lane == 0) {
      if (m_need) front = atomicAdd(count, __popcll(m_need));
      if (m_rest) back = atomicAdd(count + 1, __popcll(m_rest));
    }
    front = __builtin_amdgcn_readfirstlane(front);
    back = __builtin_amdgcn_readfirstlane(back);
    if (need) order[front + __popcll(m_need & below)] = int32_t(t);
    else if (in) order[T - 1 - (back + __popcll(m_rest & below))] = int32_t(t);
  }
}

// Long rows that a CU holds: kStreamVecs vectors per thread of 1024, the first kStreamLds of them in LDS, in slots of the wave's own that
// are filled by direct loads: as soon as a slot has been turned into gradient it is asked to be filled with the next row's vector, so
// that a CU reads while it writes.  Nothing in the row's course may wait for the stores under way, which a wait for any load behind them
// does: the next row's list, its places and sums are looked after while this row's registers fill, between the sums over the
// slots and over the registers, and no loaded register is carried from one row to the next.  (With the list at the top of its own
// row: 885 us for 8192 x 151936 bf16.)
constexpr int kStreamNT = 1024, kStreamVecs = 20, kStreamLds = 9;
constexpr int kStreamLdsBytes = kStreamLds * kStreamNT * 16;
template <int DT>
__global__ __launch_bounds__(kStreamNT) void k_distill_stream(DistillArgs a, const float* __restrict__ weight,
                                                               const int32_t* __restrict__ order) {
  using View = RowView<DT, true>;
  constexpr int E = View::E, NT = kStreamNT, NL = kStreamLds, NR = kStreamVecs - kStreamLds;
  __shared__ ListPlaces<NT> lists[2];          // by the row's parity, like everything below
  __shared__ SoftTotal s_sum[2][NT / kWave];
  __shared__ ListSums s_list[2][kListWaves];
  __shared__ int s_twice[2][kListWaves];
  extern __shared__ __align__(16) u32x4_t slots_raw[];   // NL x NT vectors
  u32x4_t(*slots)[NT] = reinterpret_cast<u32x4_t(*)[NT]>(slots_raw);
  const int tid = threadIdx.x, wave = tid / kWave, K = a.K, list_waves = (K + kWave - 1) / kWave;
  const bool lister = wave < list_waves;   // uniform in a wave
  const uint32_t voff = uint32_t(tid) * 16u;
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  auto fill_slot = [&](__amdgpu_buffer_rsrc_t src, int u) {   // lane l of wave w lands at slots[u][64 w + l]
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, &slots[u][(tid >> 6) << 6], 16, voff + uint32_t(u) * (NT * 16u), 0, 0, 2);
  };
  auto row_at = [&](int64_t p) -> int64_t { return p < a.T ? int64_t(order[p]) : a.T; };
  auto weight_of = [&](int64_t t) { return t < a.T ? weight[t] : 0.f; };
  // a lister's entry of a row: place, probability; its logit is on its way
  auto take = [&](ListPlaces<NT>& list, const View& row, int j, float lp, ListEntry& entry, bool& bad, uint32_t& raw) {
    if (tid >= K) j = -1;
    bad = j >= a.V;
    if (bad) j = -1;
    entry = ListEntry{j, 0.0, double(lp), 0.f};
    raw = load_raw<DT>(row.row, max(j, 0));
    if (j >= 0) {
      list_place(list, row, tid, j);
      entry.p = list_prob(lp);
      list.p[tid] = float(entry.p);
    }
  };

  // rows with a weight, which are alike in their cost, come first, then those that are only zeroed: every gridDim.x-th is this
  // workgroup's; p: position of the next row
  int64_t p = blockIdx.x;
  int64_t t = row_at(p);
  p += gridDim.x;
  lists[0].head[tid] = -1;
  lists[1].head[tid] = -1;
  __syncthreads();
  float w = weight_of(t);
  bool have = false;   // this thread has an entry of the row's list
  if (w != 0.f) {
    const View row(a.logits, t, a.ld, a.V);
    if (lister) {
      ListEntry entry;
      bool bad;
      uint32_t raw;
      const int k = min(tid, K - 1);
      take(lists[0], row, a.index[t * K + k], a.logprob[t * K + k], entry, bad, raw);
      entry.z = widen<DT>(raw);
      if (entry.j >= 0) lists[0].z[tid] = entry.z;
      list_sum(entry, bad, s_list[0]);
      have = entry.j >= 0;
    }
    const __amdgpu_buffer_rsrc_t src = row.buffer(row.row);
#pragma unroll
    for (int u = 0; u < NL; ++u) fill_slot(src, u);
  }
  __syncthreads();
  for (int par = 0; t < a.T; par ^= 1) {
    ListPlaces<NT>& list = lists[par];
    const int64_t tn = row_at(p);
    const View row(a.logits, t, a.ld, a.V);
    const int nvec = row.nvec, jr = row.ragged();
    char* const drow = row_ptr<DT>(a.dlogits, t, a.ld);
    const float wn = weight_of(tn);
    const View nrow(a.logits, wn != 0.f ? tn : t, a.ld, a.V);
    const __amdgpu_buffer_rsrc_t nsrc = nrow.buffer(nrow.row), dst = row.buffer(drow);
    bool zeros = true;
    if (w != 0.f) {   // uniform
      const int64_t at = (wn != 0.f ? tn : t) * K + min(tid, K - 1);
      const int jn = a.index[at];
      const float lpn = a.logprob[at];
      const uint32_t zraw = load_raw<DT>(row.row, max(jr, 0));
      const __amdgpu_buffer_rsrc_t src = row.buffer(row.row);
      uint32_t voff_ld = voff;
      asm volatile("" : "+v"(voff_ld));   // offsets are formed per row: hoisted out of the loop they are twenty registers
      u32x4_t v[NR];
#pragma unroll
      for (int u = 0; u < NR; ++u) v[u] = __builtin_amdgcn_raw_buffer_load_b128(src, voff_ld + uint32_t(NL + u) * (NT * 16u), 0, 2);
      if (lister) {
        const bool twice = have && list_twice(list, tid);
        const uint64_t any = __builtin_amdgcn_ballot_w64(twice);
        if (tid % kWave == 0) s_twice[par][wave] = any != 0;
      }
      const PlaceBits<kStreamVecs, E> listed(list);
      // Loads return in order and the NR of the registers were issued behind those into this wave's slots: with no more than NR
      // outstanding the slots have landed (the compiler does not track them; other accesses only make the wait longer).
      static_assert(NR <= 15, "immediate below holds vmcnt in 4 bits");
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0F70 | NR);
      asm volatile("" ::: "memory");
      SoftSum st = soft_identity();
      auto fold = [&](const u32x4_t& x, int u) {
        float z[E];
        View::unpack(x, z);
        listed.mask(z, u);
        soft_update<E>(st, z);
      };
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        if (tid < nvec - u * NT) fold(slots[u][tid], u);
        __builtin_amdgcn_sched_barrier(0);   // one vector at a time: keeps temporaries from piling up
      }
      ListEntry entry{-1, 0.0, 0.0, 0.f};
      bool bad = false;
      uint32_t raw = 0;
      if (lister && wn != 0.f) take(lists[par ^ 1], nrow, jn, lpn, entry, bad, raw);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < NR; ++u) {
        if (tid < nvec - (NL + u) * NT) fold(v[u], NL + u);
        __builtin_amdgcn_sched_barrier(0);
      }
      const float zr = widen<DT>(zraw);
      if (jr >= 0) {
        float z[1] = {listed.ragged ? -INFINITY : zr};
        soft_update<1>(st, z);
      }
      if (lister && wn != 0.f) {
        entry.z = widen<DT>(raw);
        if (entry.j >= 0) lists[par ^ 1].z[tid] = entry.z;
        list_sum(entry, bad, s_list[par ^ 1]);
      }
      have = entry.j >= 0;
      const SoftTotal rest = soft_block_total<NT>(st, s_sum[par]);   // its barrier also orders loads before stores over them
      bool twice = false;
      for (int k = 0; k < list_waves; ++k) twice |= s_twice[par][k] != 0;
      const RowGrad r = row_terms(a, t, w, rest, s_list[par], list_waves, twice);
      if (!r.quiet) {
        zeros = false;
        uint32_t voff_st = voff;
        asm volatile("" : "+v"(voff_st));
        auto turned = [&](const u32x4_t& x, int u) {
          float z[E], d[E];
          View::unpack(x, z);
          grad_elts<E>(z, d, r);
          __builtin_amdgcn_raw_buffer_store_b128(pack_vec<DT>(d), dst, voff_st + uint32_t(u) * (NT * 16u), 0, 2);
        };
#pragma unroll
        for (int u = 0; u < NL; ++u) {   // LDS part first: each slot is filled again right after its last use
          const u32x4_t x = slots[u][tid];
          if (tid < nvec - u * NT) turned(x, u);
          asm volatile("" ::: "memory");
          if (wn != 0.f) fill_slot(nsrc, u);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < NR; ++u) {
          if (tid < nvec - (NL + u) * NT) turned(v[u], NL + u);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (jr >= 0) store_elt<DT>(drow, jr, r.at_other * exp2_fast(fmaf(zr, kLog2e, -r.o_rest)));
        put_listed(list, row, r, drow, jr);
      }
    } else if (tid == 0) {
      put_loss(a, t, w, 0.f);
    }
    if (zeros) {
      __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): every read of this row's slots has returned
      asm volatile("" ::: "memory");
      if (wn != 0.f) {
#pragma unroll
        for (int u = 0; u < NL; ++u) fill_slot(nsrc, u);
      }
      for (int i = tid; i < nvec; i += NT) __builtin_amdgcn_raw_buffer_store_b128(zero, dst, uint32_t(i) * 16u, 0, 2);
      if (jr >= 0) store_elt<DT>(drow, jr, 0.f);
    }
    list.head[tid] = -1;   // for the row after the next
    // what is placed and written before the next row's reduction may still be read here; stores need not have landed
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    t = tn;
    w = wn;
    p += gridDim.x;
  }
}

// Fixed order, 64-bit sums.
constexpr int kSumNT = 1024;
__global__ __launch_bounds__(kSumNT) void k_distill_sum(const float* __restrict__ term, int64_t T, float* __restrict__ loss) {
  __shared__ double lds[kSumNT / kWave];
  constexpr int kAhead = 8;
  double acc = 0.0;
  for (int64_t t0 = threadIdx.x; t0 < T; t0 += kAhead * kSumNT) {
    float x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = t0 + u * kSumNT < T ? term[t0 + u * kSumNT] : 0.f;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) acc += double(x[u]);
  }
  acc = wave_sum_d(acc);
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = acc;
  __syncthreads();
  if (threadIdx.x >= kWave) return;
  acc = wave_sum_d(threadIdx.x < kSumNT / kWave ? lds[threadIdx.x] : 0.0);
  if (threadIdx.x == 0) loss[0] = float(acc);
}

struct DistillWorkspace {
  float* term;      // [T]
  int32_t* order;   // [T]
  int32_t* ctr;     // [2]
  RowSplit* split;  // [rows that are split]
  size_t bytes;
};
static DistillWorkspace distill_workspace(void* base, int64_t T) {
  const size_t each = (size_t(T) * 4 + 255) / 256 * 256, split = std::min<int64_t>(T, compute_units()) * sizeof(RowSplit);
  char* const p = reinterpret_cast<char*>(base);
  return DistillWorkspace{reinterpret_cast<float*>(p), reinterpret_cast<int32_t*>(p + each), reinterpret_cast<int32_t*>(p + 2 * each),
                          reinterpret_cast<RowSplit*>(p + 2 * each + 256), 2 * each + 256 + (split + 255) / 256 * 256};
}
size_t distill_workspace_bytes(int64_t T, int32_t V) {
  (void)V;
  return distill_workspace(nullptr, T).bytes;
}

// Workgroups that a row is split over, two to a CU in all: few rows that threads of one workgroup cannot hold in registers, and those that a CU cannot
// hold up to one per CU.  (151936 bf16, whole / 4 / 8 / 16 parts: 16 rows 25.2 / 18.0 / 13.6 / 12.2 us, 64 26.3 / 18.7 / 16.1 / 17.0, 128 28.8 / 26.4 / 25.7 /
// 29.2, 200 31.6 / 36.7 / 34.3 / 39.0; 151936 fp32 64 rows 50.7 / 25.2 / 22.4 / 22.4, 200 66.6 / 60.7 / 57.3 / 58.2; 50257 bf16, held in
// registers, 16 rows 12.0 / 11.5 / 11.4 / 11.5.)
static int distill_parts(const DistillArgs& a, bool vec, int nvec, int NT) {
  const int cus = compute_units();
  const bool held = vec && nvec <= kHeldVecs * 1024, streams = vec && a.dlogits && nvec <= kStreamVecs * kStreamNT;
  if (held || a.T > (streams ? cus / 2 : cus)) return 1;
  return int(std::max<int64_t>(1, std::min<int64_t>({kMaxParts, 2 * cus / a.T, nvec / (2 * NT)})));
}

template <int NT, int DT> static void held_launch(const DistillArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_distill_held<NT, DT>), dim3(unsigned(a.T)), dim3(NT), 0, s, a);
}

template <int DT> static aero_status distill_launch(const DistillArgs& a, bool vec, const DistillWorkspace& ws, hipStream_t s) {
  const int nvec = vec ? a.V / Storage<DT>::kPerVec : a.V;
  constexpr int NT = 512;
  const int parts = distill_parts(a, vec, nvec, NT);
  if (parts > 1) {
    const dim3 grid{unsigned(a.T), unsigned(parts)};
    const auto sums = vec ? k_distill_row<kSums, NT, DT, true> : k_distill_row<kSums, NT, DT, false>;
    const auto grad = vec ? k_distill_row<kGradient, NT, DT, true> : k_distill_row<kGradient, NT, DT, false>;
    hipLaunchKernelGGL(sums, grid, dim3(NT), 0, s, a, parts, ws.split);
    hipLaunchKernelGGL(grad, a.dlogits ? grid : dim3(unsigned(a.T)), dim3(NT), 0, s, a, parts, ws.split);
  } else if (!vec) {
    hipLaunchKernelGGL((k_distill_row<kWhole, NT, DT, false>), dim3(unsigned(a.T)), dim3(NT), 0, s, a, parts, ws.split);
  } else if (nvec > kStreamVecs * kStreamNT || (!a.dlogits && nvec > kHeldVecs * 1024)) {
    hipLaunchKernelGGL((k_distill_row<kWhole, NT, DT, true>), dim3(unsigned(a.T)), dim3(NT), 0, s, a, parts, ws.split);
  } else if (nvec <= kHeldVecs * 64 && a.K <= 64) {
    held_launch<64, DT>(a, s);
  } else if (nvec <= kHeldVecs * 256) {
    held_launch<256, DT>(a, s);
  } else if (nvec <= kHeldVecs * 512) {
    held_launch<512, DT>(a, s);
  } else if (nvec <= kHeldVecs * 1024) {
    held_launch<1024, DT>(a, s);
  } else {
    // raising the limit of dynamic LDS is per function; done once per process, safely from any thread
    static std::once_flag once;
    static hipError_t rc = hipSuccess;
    std::call_once(once, [] {
      rc = hipFuncSetAttribute(reinterpret_cast<const void*>(k_distill_stream<DT>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               kStreamLdsBytes);
    });
    if (rc != hipSuccess) return AERO_ERR_HIP;
    const unsigned grid = unsigned(std::min<int64_t>(a.T, compute_units()));
    if (a.T <= 8 * kOrderNT) {
      hipLaunchKernelGGL(k_distill_order<true>, dim3(1), dim3(kOrderNT), 0, s, a.T, a.weight, ws.ctr, ws.order);
    } else {
      hipLaunchKernelGGL(k_distill_start, dim3(1), dim3(2), 0, s, ws.ctr);
      hipLaunchKernelGGL(k_distill_order<false>, dim3(unsigned((a.T + kOrderNT - 1) / kOrderNT)), dim3(kOrderNT), 0, s, a.T, a.weight, ws.ctr,
                         ws.order);
    }
    hipLaunchKernelGGL(k_distill_stream<DT>, dim3(grid), dim3(kStreamNT), kStreamLdsBytes, s, a, a.weight, ws.order);
  }
  return AERO_OK;
}

}  // namespace aero

extern "C" aero_status aero_distill_loss_bwd(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                             const int32_t* teacher_index, const float* teacher_logprob, int32_t K,
                                             const float* token_weight, int32_t tail, float grad_scale, float* loss, float* row_loss,
                                             void* dlogits, int32_t* err_flag, void* workspace, size_t workspace_bytes,
                                             void* stream) {
  using namespace aero;
  if (T < 0 || V < 1 || V > (1 << 24) || ld < V || K < 1 || !grid_fits(T, 1024)) return AERO_ERR_SHAPE;
  if (K > kListMax) return AERO_ERR_LIMIT;
  if (tail != AERO_TAIL_RENORM && tail != AERO_TAIL_BUCKET) return AERO_ERR_SHAPE;
  if (grad_scale != grad_scale) return AERO_ERR_SHAPE;
  if (!storage_dtype_ok(dtype)) return AERO_ERR_DTYPE;
  if (!loss) return AERO_ERR_NULL;
  if (T > 0 && (!logits || !teacher_index || !teacher_logprob || !token_weight)) return AERO_ERR_NULL;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < distill_workspace_bytes(T, V))
    return AERO_ERR_WORKSPACE;
  const hipStream_t s = as_stream(stream);
  const DistillWorkspace ws = distill_workspace(workspace, T);
  const DistillArgs a{logits, T, V, ld, teacher_index, teacher_logprob, K, token_weight, tail, grad_scale, ws.term, row_loss, dlogits, err_flag};
  if (T > 0) {
    const bool vec = rows_alike(logits, dlogits, storage_bytes(dtype));
    const aero_status st = dtype == AERO_BF16 ? distill_launch<kBF16>(a, vec, ws, s) : dtype == AERO_F16 ? distill_launch<kF16>(a, vec, ws, s)
                           : dtype == AERO_F8E4M3 ? distill_launch<kF8>(a, vec, ws, s) : distill_launch<kF32>(a, vec, ws, s);
    if (st != AERO_OK) return st;
  }
  hipLaunchKernelGGL(k_distill_sum, dim3(1), dim3(kSumNT), 0, s, a.term, T, loss);
  return launch_status();
}
