// Rows of logits that may be masked: their log-partition, and walks over their vectors that a workgroup or a part of
// one makes.  Shared by the calls around a drafter (top-K lists, distillation, verification).
#pragma once
#include <type_traits>

#include "aero_device.h"

namespace aero {

// A logit at or below this is masked (-inf, the lowest value of fp32 or bf16, -1e10, as masks write it); one at or above its negative makes the row NaN, as
// +inf does.  In between an offset of 32 bits, whose unit is at most 128, is within 64 of its logit's z log2 e, so that no exponential that is kept
// overflows, or vanishes beside its own offset; beyond (z = -1e10: 440 off) sums would be inf or 0.
constexpr float kMasked = -AERO_LOGIT_LIMIT, kTooLarge = AERO_LOGIT_LIMIT;
// Where a running offset starts, in units of log 2: the largest masked logit's exponent is 234 below it, so that those of masked logits are 0 by
// themselves, and the smallest other one's (128 more, the logits' own unit there) 49 below.
constexpr float kMaskedLog2 = -1731233792.f;
static_assert(AERO_LOGIT_LIMIT == 1.2e9f, "kMaskedLog2 goes with it");

// 2^o s = sum of 2^(z log2 e) over the logits, o a whole number near the largest z log2 e.  Being whole, it is subtracted inside the fused
// multiply-add without a rounding of its own, and sums with different offsets meet without one either: the error of an exponential is
// that of its argument near the offset, whatever the size of the logits up to 2^23 (and 2^-18 up to the limit).  (An offset in the logits' own units costs
// 2^-24 |z| in every probability, 3 times the error of a gradient in fp32.)  s == 0: nothing but masked logits.  A NaN or too large logit
// makes s NaN.
struct SoftSum {
  float o, s;
};
__device__ __forceinline__ SoftSum soft_identity() { return SoftSum{kMaskedLog2, 0.f}; }
// The offset for a logit; NaN where it is too large, which makes s, and whatever the sum meets, NaN.
__device__ __forceinline__ float soft_offset(float z) { return z < kTooLarge ? rintf(z * kLog2e) : __builtin_nanf(""); }

// The largest of a vector's logits (NaN are passed over).
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

// The offset moves only for a logit more than 2^kAbove above it, so the rescaling is rare (the test in front and the side effect keep it a
// branch, see stat_update).
constexpr float kAbove = 17.f;
__device__ __forceinline__ void soft_grow(SoftSum& st, float vm) {
  const bool grow = fmaf(vm, kLog2e, -st.o) > kAbove;
  if (__builtin_amdgcn_ballot_w64(grow) != 0) {
    asm volatile("" ::: "memory");
    if (grow) {
      const float o = soft_offset(vm);
      st.s *= exp2_fast(st.o - o);
      st.o = o;
    }
  }
}
template <int N> __device__ __forceinline__ void soft_add(SoftSum& st, const float (&z)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) st.s += exp2_fast(fmaf(z[k], kLog2e, -st.o));
}
template <int N> __device__ __forceinline__ void soft_update(SoftSum& st, const float (&z)[N], float vm) {
  soft_grow(st, vm);
  soft_add<N>(st, z);
}
template <int N> __device__ __forceinline__ void soft_update(SoftSum& st, const float (&z)[N]) { soft_update<N>(st, z, vec_max<N>(z)); }

__device__ __forceinline__ SoftSum soft_rescaled(SoftSum a, float o) {
  return SoftSum{o, a.o == o ? a.s : a.s * exp2_fast(a.o - o)};
}
__device__ __forceinline__ SoftSum soft_merge(SoftSum a, SoftSum b) {
  const float o = fmaxf(a.o, b.o);
  return SoftSum{o, soft_rescaled(a, o).s + soft_rescaled(b, o).s};
}
template <bool WAVE> __device__ __forceinline__ SoftSum soft_reduce(SoftSum a) {
  auto all = [](float x, auto op) { return WAVE ? wave_reduce(x, op) : row16_reduce(x, op); };
  const float o = all(a.o, [](float x, float y) { return fmaxf(x, y); });
  return SoftSum{o, all(soft_rescaled(a, o).s, [](float x, float y) { return x + y; })};
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

// The same with the sums of the threads added up in 64 bits: what is left of an error is their own, which differs from thread to thread and
// evens out, where the last few of 32-bit additions do not.
struct SoftTotal {
  float o;
  double s;
};
__device__ __forceinline__ SoftTotal soft_total(SoftSum a) { return SoftTotal{a.o, double(a.s)}; }
__device__ __forceinline__ double soft_rescaled(SoftTotal a, float o) { return a.s * double(exp2_fast(a.o - o)); }
__device__ __forceinline__ SoftTotal soft_merge(SoftTotal a, SoftTotal b) {
  const float o = fmaxf(a.o, b.o);
  return SoftTotal{o, soft_rescaled(a, o) + soft_rescaled(b, o)};
}
// Over 16 lanes in a row.
__device__ __forceinline__ double row16_sum_d(double v) {
  const auto moved = [](auto ctrl, double x) {
    return __hiloint2double(dpp_move_i<ctrl.value>(__double2hiint(x)), dpp_move_i<ctrl.value>(__double2loint(x)));
  };
  v += moved(std::integral_constant<int, 0xB1>{}, v);
  v += moved(std::integral_constant<int, 0x4E>{}, v);
  v += moved(std::integral_constant<int, 0x141>{}, v);
  return v + moved(std::integral_constant<int, 0x140>{}, v);
}
template <bool WAVE> __device__ __forceinline__ SoftTotal soft_reduce(SoftTotal a) {
  const auto most = [](float x, float y) { return fmaxf(x, y); };
  const float o = WAVE ? wave_reduce(a.o, most) : row16_reduce(a.o, most);
  const double s = soft_rescaled(a, o);
  return SoftTotal{o, WAVE ? wave_sum_d(s) : row16_sum_d(s)};
}
template <int NT> __device__ __forceinline__ SoftTotal soft_block_total(SoftSum mine, SoftTotal* lds /*[NT/64]*/) {
  SoftTotal a = soft_reduce<true>(soft_total(mine));
  constexpr int kWaves = NT / kWave;
  static_assert(kWaves <= 16, "one lane per wave in the second step");
  if constexpr (kWaves > 1) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (lane == 0) lds[wave] = a;
    __syncthreads();
    a = soft_reduce<false>(lane % 16 < kWaves ? lds[lane % 16] : soft_total(soft_identity()));
  }
  return a;
}

// e^x for a 32-bit x, or a 64-bit one within +-800, in 64 bits: 2^n e^r with |r| <= ln 2 / 2 and the exponential series up to r^11 / 11! (the next term is under
// 1e-14; what a list leaves of 1 may be 1e-8, of which r^8 / 8! as the last one leaves two digits).  The coefficients behind r^7 in 32 bits: their
// roundings are under 1e-16 of the sum.
__device__ __forceinline__ double exp_of(double x) {
  const float n = rintf(float(x) * kLog2e);
  const double r = fma(double(n), -0.69314718055994531, x);
  const float f = float(r);
  double y = double(fmaf(fmaf(fmaf(1.f / 39916800, f, 1.f / 3628800), f, 1.f / 362880), f, 1.f / 40320));
  y = fma(y, r, 1.0 / 5040);
  y = fma(y, r, 1.0 / 720);
  y = fma(y, r, 1.0 / 120);
  y = fma(y, r, 1.0 / 24);
  y = fma(y, r, 1.0 / 6);
  y = fma(y, r, 0.5);
  y = fma(y, r, 1.0);
  return ldexp(fma(y, r, 1.0), int(n));
}
// Logarithm of a positive number x = 2^k f, f in [1/sqrt 2, sqrt 2), in 64 bits: of f's 32-bit rounding, whose logarithm rounds by 2^-26 at most, and
// of what that leaves.
__device__ __forceinline__ double log_of(double x) {
  double f = __builtin_amdgcn_frexp_mant(x);
  int k = __builtin_amdgcn_frexp_exp(x);
  if (f < 0.70710678) {
    f *= 2.0;
    --k;
  }
  const float g = float(f);
  return double(k) * 0.69314718055994531 + (double(logf(g)) + double(float(f - double(g)) / g));
}
// log sum exp in 64 bits: (o + log2 s) / log2 e; log2 e is the rounded one that the sums were formed with.  -inf for an empty row, NaN for one with a
// NaN or too large logit.
__device__ __forceinline__ double soft_lse(SoftTotal st) {
  if (st.s == 0.0) return -INFINITY;
  const double lse = (double(st.o) + log_of(st.s) * 1.4426950408889634) * (1.0 / double(kLog2e));
  return st.s == st.s ? lse : __builtin_nan("");
}
__device__ __forceinline__ double soft_lse(SoftSum st) { return soft_lse(soft_total(st)); }

// Inclusive sums over the lanes of a wave, lane by lane in the registers (LDS is not taken).
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  const auto plus = [&](auto ctrl, auto rows) { x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), ctrl.value, rows.value, 0xf, true)); };
  plus(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // 1, 2, 4, 8 lanes along a row of 16
  plus(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  plus(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  plus(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  plus(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // a row's last lane to the row behind it
  plus(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // the first half's last lane to the second half
  return x;
}

// An element as it is stored, to be widened where it is needed: a conversion next to the load waits for it there.
template <int DT> __device__ __forceinline__ uint32_t load_raw(const char* row, int j) {
  if constexpr (Storage<DT>::kBytes == 2) return reinterpret_cast<const uint16_t*>(row)[j];
  else if constexpr (Storage<DT>::kBytes == 1) return reinterpret_cast<const uint8_t*>(row)[j];
  else return reinterpret_cast<const uint32_t*>(row)[j];
}
template <int DT> __device__ __forceinline__ float widen(uint32_t raw) {
  if constexpr (DT == kBF16) return bf16_to_f32(uint16_t(raw));
  else if constexpr (DT == kF16) return f16_to_f32(uint16_t(raw));
  else if constexpr (DT == kF8) return f8_to_f32(uint8_t(raw));
  else return __uint_as_float(raw);
}

// 16 bytes, or four floats, at any element's alignment: the same instructions, which the machine takes at any address.
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(1)));
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));

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
  // the same for a vector that was read before: out of the caches
  __device__ __forceinline__ u32x4_t load_again(int vec) const {
    if constexpr (VEC) return reinterpret_cast<const u32x4_t*>(row + head * Storage<DT>::kBytes)[vec];
    else return load(vec);
  }
  __device__ __forceinline__ static void unpack(const u32x4_t& v, float (&z)[E]) {
    if constexpr (VEC) unpack_vec<DT>(v, z);
    else z[0] = __uint_as_float(v.x);
  }
  // the vectors as a buffer, whose bounds check returns zeros (and drops stores) behind the last one
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const char* base) const {
    static_assert(VEC, "of 16-byte vectors");
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base) + head * Storage<DT>::kBytes, 0, nvec * 16, 0x00020000);
  }
  __device__ __forceinline__ float at(int j) const { return load_elt<DT>(row, j); }
  // the element outside the vectors that this thread looks after, -1: none
  __device__ __forceinline__ int ragged() const {
    if constexpr (VEC) return ragged_elt<DT>(RowGeom{head, nvec}, V, threadIdx.x);
    else return -1;
  }
};

}  // namespace aero
