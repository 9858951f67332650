// Rows of logits that may be masked: their log-partition, and walks over their vectors that a workgroup or a part of
// one makes.  Shared by the calls around a drafter (top-K lists, distillation, verification).
#pragma once
#include "aero_device.h"

namespace aero {

// A logit at or below this is masked (-inf, or the lowest value of fp32 / bf16, as masks write it).  It is also where a running
// offset starts: exp(z - offset) of a masked logit is then 0 by itself, and never inf - inf.
constexpr float kMasked = -1e30f;

// Sum of exp(z - m) with an offset m that is near the largest z.  s == 0: nothing but masked logits.  A NaN or +inf logit makes
// s NaN.
struct SoftSum {
  float m, s;
};
__device__ __forceinline__ SoftSum soft_identity() { return SoftSum{kMasked, 0.f}; }

// The offset moves only for a logit more than kLazy above it (see stat_update, whose sums these are without the third one).
template <int N> __device__ __forceinline__ float vec_max(const float (&z)[N]) {
  float vm = z[0];
  if constexpr (N >= 3) {
#pragma unroll
    for (int k = 1; k + 1 < N; k += 2) vm = max3(vm, z[k], z[k + 1]);
    if constexpr (N % 2 == 0) vm = fmaxf(vm, z[N - 1]);
  } else if constexpr (N == 2) {
    vm = fmaxf(vm, z[1]);
  }
  return vm;
}
template <int N> __device__ __forceinline__ void soft_update(SoftSum& st, const float (&z)[N], float vm) {
  const bool grow = vm > st.m + kLazy;
  if (__builtin_amdgcn_ballot_w64(grow) != 0) {
    asm volatile("" ::: "memory");   // a side effect: the block cannot be if-converted
    if (grow) {
      st.s *= exp2_fast((st.m - vm) * kLog2e);
      st.m = vm;
    }
  }
  const float c = -st.m * kLog2e;
#pragma unroll
  for (int k = 0; k < N; ++k) st.s += exp2_fast(fmaf(z[k], kLog2e, c));
}
template <int N> __device__ __forceinline__ void soft_update(SoftSum& st, const float (&z)[N]) { soft_update<N>(st, z, vec_max<N>(z)); }

__device__ __forceinline__ SoftSum soft_rescaled(SoftSum a, float M) {
  return SoftSum{M, a.m == M ? a.s : a.s * exp2_fast((a.m - M) * kLog2e)};
}
__device__ __forceinline__ SoftSum soft_merge(SoftSum a, SoftSum b) {
  const float M = fmaxf(a.m, b.m);
  return SoftSum{M, soft_rescaled(a, M).s + soft_rescaled(b, M).s};
}
template <bool WAVE> __device__ __forceinline__ SoftSum soft_reduce(SoftSum a) {
  auto all = [](float x, auto op) { return WAVE ? wave_reduce(x, op) : row16_reduce(x, op); };
  const float M = all(a.m, [](float x, float y) { return fmaxf(x, y); });
  return SoftSum{M, all(soft_rescaled(a, M).s, [](float x, float y) { return x + y; })};
}
// Over the workgroup, every thread gets the result; one barrier.  lds is free again after the next barrier.
template <int NT> __device__ __forceinline__ SoftSum soft_block_reduce(SoftSum a, SoftSum* lds /*[NT/64]*/) {
  a = soft_reduce<true>(a);
  constexpr int kWaves = NT / kWave;
  static_assert(kWaves <= 16, "one lane per wave in the second step");
  if constexpr (kWaves > 1) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (lane == 0) lds[wave] = a;
    __syncthreads();
    a = soft_reduce<false>(lane % 16 < kWaves ? lds[lane % 16] : soft_identity());
  }
  return a;
}

// Log-partition, log-prob of a logit zy of the row and its rounding remainder.  An empty row: lse -inf, log-probs NaN.
__device__ __forceinline__ RowLogProb soft_logprob(SoftSum st, float zy) {
  if (st.s == 0.f) return RowLogProb{-INFINITY, __builtin_nanf(""), 0.f};
  return row_logprob(RowStat{st.m, st.s, 0.f}, zy);
}

// One row as E-element vectors (VEC: 16 bytes between the ragged ends; otherwise single elements), of which this workgroup looks
// after [first, last); the ragged ends belong to the part that starts at 0.
template <int DT, bool VEC> struct RowView {
  static constexpr int E = VEC ? Storage<DT>::kPerVec : 1;
  const char* row;
  int head, nvec, V;

  __device__ __forceinline__ RowView(const void* base, int64_t t, int64_t ld, int v) : row(row_ptr<DT>(base, t, ld)), V(v) {
    const RowGeom g = VEC ? row_geom<DT>(base, t, ld, v) : RowGeom{0, v};
    head = g.head;
    nvec = g.nvec;
  }
  __device__ __forceinline__ int column(int vec) const { return head + vec * E; }
  // raw vector: 16 bytes, or an element widened to fp32 in .x
  __device__ __forceinline__ u32x4_t load(int vec) const {
    if constexpr (VEC) {
      return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + head * Storage<DT>::kBytes) + vec);
    } else {
      return u32x4_t{__float_as_uint(load_elt<DT>(row, vec)), 0u, 0u, 0u};
    }
  }
  __device__ __forceinline__ static void unpack(const u32x4_t& v, float (&z)[E]) {
    if constexpr (VEC) unpack_vec<DT>(v, z);
    else z[0] = __uint_as_float(v.x);
  }
  __device__ __forceinline__ float at(int j) const { return load_elt<DT>(row, j); }
  // the element outside the vectors that this thread looks after, -1: none
  __device__ __forceinline__ int ragged() const {
    if constexpr (VEC) return ragged_elt<DT>(RowGeom{head, nvec}, V, threadIdx.x);
    else return -1;
  }
};

}  // namespace aero
