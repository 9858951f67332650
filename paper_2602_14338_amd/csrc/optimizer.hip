// What happens to gradients: their norm over many tensors, and Adam's step with decoupled weight decay on all of them at once, with moments
// in 32 bits or in 8.
//
// A table describes the tensors.  Its elements are dealt out in chunks of 2048 of one tensor; the chunks of tensors of one class (types of
// parameter, gradient and moments) stand together, and a class is one launch.
//
// Bound by bytes: n of the gradient for the norm (500 M bf16 154 us, 6.5 TB/s), for a step what is read and written of weights and moments (28 bytes an element for 16-bit weights with
// a master and 32-bit moments: 300 M 1351 us, 6.2 TB/s).  With 8-bit moments (10 bytes an element) a step is bound by vector instructions, 99 an element where it rounds at random: 233 M
// 550-600 us, of which the bytes are 370.  Small ones by one launch: 262 K elements 4.3 us, the norm of 150 K 4.0.
#include <cmath>
#include <cstring>

#include "row_scan.h"

namespace aero {

// ---------------------------------------------------------------------------------- the table
constexpr int kOptNT = 256, kChunk = 2048, kBlock = AERO_MOMENT_BLOCK;
// Elements of a lane, side by side: of 32-bit arrays four, 16 bytes; eight where moments are codes, so that half a wave holds a block of them.
constexpr int kWideLane = 4, kCodeLane = 8;
static_assert(kBlock == kWave / 2 * kCodeLane && kChunk == kOptNT * kCodeLane, "a chunk is blocks of half a wave each");

enum ParamKind { kNoParam, kParamF32, kParamBF16, kMasterBF16, kMasterF16, kParamKinds };
constexpr int kGrads = 3, kClasses = kParamKinds * kGrads * 2;   // times the gradient's type, times the moments'
constexpr int class_of(int param, int grad, int bits8) { return (param * kGrads + grad) * 2 + bits8; }

struct Tensor {
  char* param;
  const char* grad;
  float* master;
  char *avg, *sq;
  float *avg_scale, *sq_scale;
  int64_t n;
  int64_t out;            // where its moments begin in aero_adamw_moments's outputs
  uint32_t first_chunk;
  int32_t ordinal;        // place in the caller's list
  float decay;
  int32_t kind;           // its class
  int64_t pad;
};
static_assert(sizeof(Tensor) % 16 == 0, "read in 16-byte pieces");

// What a step has worked out before it looks at an element.
struct StepScalars {
  float factor, by_first, by_second;
  uint32_t of_step;       // the random bits' part of seed and step
  double weight_decay;    // times the rate
};

// Workgroups of a small launch count themselves off as they end, so that the last one knows: in sixteen groups first, each on a cache line of its own, as
// counts on one line follow each other 13 ns apart.  All are 0 again when it is over.
constexpr int kTicketGroups = 16;
struct Tickets {
  uint32_t group[kTicketGroups][32];
  uint32_t all[32];
};

constexpr uint64_t kMagic = 0x41455254'61626c65ull;
struct Table {
  uint64_t magic;
  uint64_t bytes;
  int32_t count;
  uint32_t chunks;
  uint32_t pad[2];
  StepScalars step;       // of the step under way (device copy)
  uint32_t class_first[kClasses + 1];   // chunks of class k: class_first[k] .. class_first[k + 1]
  uint32_t pad2[3];
  Tickets step_tickets, norm_tickets;   // (device copy)
};
static_assert(sizeof(Table) % 16 == 0, "the tensors behind it are aligned");
inline size_t map_offset(int32_t count) { return sizeof(Table) + size_t(count) * sizeof(Tensor); }
__host__ __device__ inline const Tensor* tensors_of(const void* table) {
  return reinterpret_cast<const Tensor*>(static_cast<const char*>(table) + sizeof(Table));
}
__host__ __device__ inline const uint32_t* map_of(const void* table, int32_t count) {
  return reinterpret_cast<const uint32_t*>(static_cast<const char*>(table) + sizeof(Table) + size_t(count) * sizeof(Tensor));
}
static const Table* table_of(const void* image) {
  const Table* t = static_cast<const Table*>(image);
  return t && t->magic == kMagic ? t : nullptr;
}

static bool grad_dtype_ok(int32_t d) { return d == AERO_F32 || d == AERO_BF16 || d == AERO_F16; }
static aero_status check_tensor(const aero_tensor& t) {
  if (t.n < 0 || t.n >= (int64_t(1) << 32)) return AERO_ERR_SHAPE;
  if (!grad_dtype_ok(t.grad_dtype)) return AERO_ERR_DTYPE;
  const auto apart = [](const void* p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size != 0; };
  if (t.n > 0 && !t.grad) return AERO_ERR_NULL;
  if (apart(t.grad, storage_bytes(t.grad_dtype))) return AERO_ERR_ALIGN;
  if (!t.param) return AERO_OK;
  if (!grad_dtype_ok(t.param_dtype) || (t.param_dtype == AERO_F16 && !t.master) || (t.param_dtype == AERO_F32 && t.master)) return AERO_ERR_DTYPE;
  if (!(t.decay - t.decay == 0.f)) return AERO_ERR_SHAPE;
  if (!t.exp_avg || !t.exp_avg_sq || !t.exp_avg_scale != !t.exp_avg_sq_scale) return AERO_ERR_NULL;
  if (apart(t.param, storage_bytes(t.param_dtype)) || apart(t.master, 4) || apart(t.exp_avg_scale, 4) || apart(t.exp_avg_sq_scale, 4)) return AERO_ERR_ALIGN;
  if (!t.exp_avg_scale && (apart(t.exp_avg, 4) || apart(t.exp_avg_sq, 4))) return AERO_ERR_ALIGN;
  return AERO_OK;
}
static int class_of(const aero_tensor& t) {
  const int grad = t.grad_dtype == AERO_F32 ? 0 : t.grad_dtype == AERO_BF16 ? 1 : 2;
  if (!t.param) return class_of(kNoParam, grad, 0);
  const int kind = t.param_dtype == AERO_F32 ? kParamF32 : t.param_dtype == AERO_F16 ? kMasterF16 : t.master ? kMasterBF16 : kParamBF16;
  return class_of(kind, grad, t.exp_avg_scale ? 1 : 0);
}
static uint64_t chunks_of(const aero_tensor& t) { return (uint64_t(t.n) + kChunk - 1) / kChunk; }

// ---------------------------------------------------------------------------------- elements
// At any alignment, and past the caches: nothing is read twice.
typedef uint32_t u32x4_at_t __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_at_t __attribute__((ext_vector_type(2), aligned(1)));

// Waits for what this wave has under way in memory, if asked to.
template <bool ASKED> __device__ __forceinline__ void arrived() {
  if constexpr (ASKED) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    asm volatile("" ::: "memory");
  }
}
// By one thread of each workgroup, behind all that the workgroup has to be known for: is it the last one?
__device__ __forceinline__ bool count_off(Tickets& t) {
  const auto count = [](uint32_t* word, uint32_t of) {
    if (atomicAdd(word, 1u) != of - 1) return false;
    *word = 0;
    return true;
  };
  const uint32_t group = blockIdx.x % kTicketGroups, n = gridDim.x;
  if (!count(t.group[group], (n - group + kTicketGroups - 1) / kTicketGroups)) return false;
  return count(t.all, n < uint32_t(kTicketGroups) ? n : uint32_t(kTicketGroups));
}
// How many of the N elements from i on a tensor of n has.
template <int N> __device__ __forceinline__ int have_of(int64_t n, uint64_t i) {
  const int64_t behind = n - int64_t(i);
  return behind >= N ? N : behind > 0 ? int(behind) : 0;
}
// N stored elements of BYTES each, as words: `have` of them are the tensor's, the others read as 0 and are not written.
template <int BYTES, int N> struct Words {
  static constexpr int kWords = BYTES * N / 4;
  static_assert(kWords == 2 || kWords == 4 || kWords == 8, "one or two vectors");
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* base, uint64_t i, int have) {
    const char* p = static_cast<const char*>(base) + i * BYTES;
    if (have >= N) {
      if constexpr (kWords == 2) {
        const u32x2_at_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_at_t*>(p));
        w[0] = v.x, w[1] = v.y;
      } else {
#pragma unroll
        for (int k = 0; k < kWords; k += 4) {
          const u32x4_at_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_at_t*>(p + 4 * k));
          w[k] = v.x, w[k + 1] = v.y, w[k + 2] = v.z, w[k + 3] = v.w;
        }
      }
      return;
    }
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = 0;
#pragma unroll
    for (int k = 0; k < N - 1; ++k) {
      if (k >= have) continue;
      if constexpr (BYTES == 4) w[k] = reinterpret_cast<const uint32_t*>(p)[k];
      else if constexpr (BYTES == 2) w[k / 2] |= uint32_t(reinterpret_cast<const uint16_t*>(p)[k]) << (16 * (k % 2));
      else w[k / 4] |= uint32_t(reinterpret_cast<const uint8_t*>(p)[k]) << (8 * (k % 4));
    }
  }
  __device__ __forceinline__ void store(void* base, uint64_t i, int have) const {
    char* p = static_cast<char*>(base) + i * BYTES;
    if (have >= N) {
      if constexpr (kWords == 2) {
        __builtin_nontemporal_store((u32x2_at_t{w[0], w[1]}), reinterpret_cast<u32x2_at_t*>(p));
      } else {
#pragma unroll
        for (int k = 0; k < kWords; k += 4)
          __builtin_nontemporal_store((u32x4_at_t{w[k], w[k + 1], w[k + 2], w[k + 3]}), reinterpret_cast<u32x4_at_t*>(p + 4 * k));
      }
      return;
    }
#pragma unroll
    for (int k = 0; k < N - 1; ++k) {
      if (k >= have) continue;
      if constexpr (BYTES == 4) reinterpret_cast<uint32_t*>(p)[k] = w[k];
      else if constexpr (BYTES == 2) reinterpret_cast<uint16_t*>(p)[k] = uint16_t(w[k / 2] >> (16 * (k % 2)));
      else reinterpret_cast<uint8_t*>(p)[k] = uint8_t(w[k / 4] >> (8 * (k % 4)));
    }
  }
};
// The same as numbers of a storage type.
template <int DT, int N> struct Numbers : Words<Storage<DT>::kBytes, N> {
  using Words<Storage<DT>::kBytes, N>::w;
  __device__ __forceinline__ void widen(float (&x)[N]) const {
    if constexpr (DT == kF32) {
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = __uint_as_float(w[k]);
    } else {
#pragma unroll
      for (int k = 0; k < N; k += 2) {
        x[k] = DT == kBF16 ? bf16_lo(w[k / 2]) : f16_to_f32(uint16_t(w[k / 2]));
        x[k + 1] = DT == kBF16 ? bf16_hi(w[k / 2]) : f16_to_f32(uint16_t(w[k / 2] >> 16));
      }
    }
  }
  __device__ __forceinline__ static void store_rounded(void* base, uint64_t i, int have, const float (&x)[N]) {
    Numbers v;
    if constexpr (DT == kF32) {
#pragma unroll
      for (int k = 0; k < N; ++k) v.w[k] = __float_as_uint(x[k]);
    } else {
#pragma unroll
      for (int k = 0; k < N; k += 2) v.w[k / 2] = DT == kBF16 ? pack_bf16x2(x[k], x[k + 1]) : pack_f16x2(x[k], x[k + 1]);
    }
    v.store(base, i, have);
  }
};
using Codes = Words<1, kCodeLane>;

// ---------------------------------------------------------------------------------- moments in 8 bits
// Codes and values as aero.h defines them; each product, sum and quotient rounded by itself (no fused multiply-add), so that the codes are a
// function of the definition alone.
constexpr float kInvTop1 = float(1.0 / 16129.0), kInvTop2 = float(1.0 / 4228250625.0);   // of 127^2, 255^4
__device__ __forceinline__ float first_value(float c, float scale) {
#pragma clang fp contract(off)
  return (c * fabsf(c)) * scale;
}
__device__ __forceinline__ float fourth(float c) {
#pragma clang fp contract(off)
  return (c * c) * (c * c);
}
__device__ __forceinline__ float second_value(float c, float scale) {
#pragma clang fp contract(off)
  return fourth(c) * scale;
}
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}
__device__ __forceinline__ float uniform16(uint32_t low16) { return fmaf(float(low16), 0x1p-16f, 0x1p-17f); }   // exact

template <bool FIRST> __device__ __forceinline__ void decode(const Codes& codes, float scale, float (&x)[kCodeLane]) {
#pragma unroll
  for (int k = 0; k < kCodeLane; ++k) {
    const uint32_t w = codes.w[k / 4] >> (8 * (k % 4));
    x[k] = FIRST ? first_value(float(int8_t(w)), scale) : second_value(float(w & 0xff), scale);
  }
}
// The scale of a block, eight of whose moments each lane of half a wave holds.  The largest by its bits: as whole numbers infinities and NaN come out largest.
template <bool SIGNED> __device__ __forceinline__ float block_scale(const float (&x)[kCodeLane], float inv_top) {
#pragma clang fp contract(off)
  auto most = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < kCodeLane; ++k) m = most(m, SIGNED ? __float_as_uint(x[k]) & 0x7fffffffu : __float_as_uint(x[k]));
  m = most(m, uint32_t(dpp_move_i<0xB1>(int(m))));
  m = most(m, uint32_t(dpp_move_i<0x4E>(int(m))));
  m = most(m, uint32_t(dpp_move_i<0x141>(int(m))));
  m = most(m, uint32_t(dpp_move_i<0x140>(int(m))));
  const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  m = most(r[0], r[1]);
  if (m >= 0x7f800000u) return __builtin_nanf("");
  const float s = __uint_as_float(m) * inv_top;
  return s >= 1.17549435e-38f ? s : 0.f;
}
// 1 / scale rounded once: the estimate is off by a unit at most, and one step with the exact remainder leaves none of it (for every mantissa, tried out).
__device__ __forceinline__ float inverse_of(float scale) {
  const float r = __builtin_amdgcn_rcpf(scale);
  return scale > 0.f ? fmaf(fmaf(-scale, r, 1.f), r, r) : 0.f;
}
// Codes of a block's moments, of which this lane has eight, in the form of aero.h but for what makes no difference:
//   - the root that a code is found by is estimated from below (kBelow: by more than the estimate's own error, 2^-22), so that the next code may be the right one
//     but the one before never is, and that rarely: a branch that few waves take;
//   - a y above the top is not cut down to it first: it rounds to at most one code more, which is cut off at the end.
// `random`: of which `shift` of the bits u is made.
constexpr float kBelow = 1.f - 0x1p-21f;
template <int SHIFT> __device__ __forceinline__ float random_or_half(bool stochastic, uint32_t bits) {
  return stochastic ? uniform16(bits >> SHIFT & 0xffff) : 0.5f;
}
__device__ __forceinline__ Codes first_codes(const float (&x)[kCodeLane], float inv, bool stochastic, const uint32_t (&bits)[kCodeLane]) {
#pragma clang fp contract(off)
  float c[kCodeLane], left[kCodeLane], step[kCodeLane];   // code, y - c^2 and (c + 1)^2 - c^2, both exact
  const float below = inv * (kBelow * kBelow);
  bool more = false;
#pragma unroll
  for (int k = 0; k < kCodeLane; ++k) {
    const float y = fabsf(x[k]) * inv;
    c[k] = floorf(__builtin_amdgcn_sqrtf(fabsf(x[k]) * below));
    left[k] = fmaf(-c[k], c[k], y);
    step[k] = fmaf(2.f, c[k], 1.f);
    more |= left[k] >= step[k];
  }
  if (__builtin_amdgcn_ballot_w64(more) != 0) {
    asm volatile("" ::: "memory");   // stays a branch
#pragma unroll
    for (int k = 0; k < kCodeLane; ++k) {
      if (left[k] >= step[k]) {
        left[k] -= step[k];
        c[k] += 1.f;
        step[k] += 2.f;
      }
    }
  }
  Codes out{};
#pragma unroll
  for (int k = 0; k < kCodeLane; ++k) {
    const float next = c[k] + 1.f;
    c[k] = __builtin_amdgcn_fmed3f(random_or_half<0>(stochastic, bits[k]) * step[k] < left[k] ? next : c[k], 0.f, 127.f);
    out.w[k / 4] |= (uint32_t(int(copysignf(c[k], x[k]))) & 0xff) << (8 * (k % 4));
  }
  return out;
}
// root: about the roots of the moments, of which a step has made use already.
__device__ __forceinline__ Codes second_codes(const float (&x)[kCodeLane], const float (&root)[kCodeLane], float inv, bool stochastic,
                                              const uint32_t (&bits)[kCodeLane]) {
#pragma clang fp contract(off)
  float y[kCodeLane], c[kCodeLane], more_c[kCodeLane], at[kCodeLane], next[kCodeLane];   // code and the next one, what they stand for
  const float below = __builtin_amdgcn_sqrtf(inv) * (kBelow * kBelow);
  bool more = false;
#pragma unroll
  for (int k = 0; k < kCodeLane; ++k) {
    y[k] = x[k] * inv;
    c[k] = floorf(__builtin_amdgcn_sqrtf(root[k] * below));
    more_c[k] = c[k] + 1.f;
    at[k] = fourth(c[k]);
    next[k] = fourth(more_c[k]);
    more |= next[k] <= y[k];
  }
  if (__builtin_amdgcn_ballot_w64(more) != 0) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < kCodeLane; ++k) {
      if (next[k] <= y[k]) {
        c[k] = more_c[k];
        at[k] = next[k];
        more_c[k] += 1.f;
        next[k] = fourth(more_c[k]);
      }
    }
  }
  Codes out{};
#pragma unroll
  for (int k = 0; k < kCodeLane; ++k) {
    const float code = random_or_half<16>(stochastic, bits[k]) * (next[k] - at[k]) < y[k] - at[k] ? more_c[k] : c[k];
    const float least = y[k] > 0.f ? 1.f : 0.f;   // a moment > 0 is not stored as 0
    out.w[k / 4] |= uint32_t(__builtin_amdgcn_fmed3f(code, least, 255.f)) << (8 * (k % 4));
  }
  return out;
}

// ---------------------------------------------------------------------------------- the step
struct StepArgs {
  void* table;
  int32_t count;
  uint32_t first, first_unit;   // chunk that this launch's class begins with; the launch's part of it
  float beta1, beta1c, beta2, beta2c, eps;
  double lr, weight_decay, dbeta1, dbeta2;
  uint32_t seed_lo, seed_hi;
  int32_t stochastic;
  int32_t* step;
  const float *factor, *lr_factor;
};

// What a lane has of a tensor, as it is stored until it is worked on, so that a wave's loads can be under way together.
template <int KIND, int GRAD, bool SMALL, bool ALONE> struct Held {
  static constexpr bool kMaster = KIND == kMasterBF16 || KIND == kMasterF16;
  static constexpr int kStored = KIND == kParamF32 ? kF32 : KIND == kMasterF16 ? kF16 : kBF16, kRead = kMaster ? kF32 : kStored;
  static constexpr int N = SMALL ? kCodeLane : kWideLane;
  static constexpr bool kOrdered = !SMALL && !ALONE;
  Numbers<GRAD, N> g;
  Numbers<kRead, N> p;
  std::conditional_t<SMALL, Codes, Numbers<kF32, N>> m, v;
  float scale_m, scale_v;

  __device__ __forceinline__ void load(const Tensor& e, uint64_t i, int have) {
    g.load(e.grad, i, have);
    arrived<kOrdered>();
    p.load(kMaster ? reinterpret_cast<const char*>(e.master) : e.param, i, have);
    arrived<kOrdered>();
    m.load(e.avg, i, have);
    arrived<kOrdered>();
    v.load(e.sq, i, have);
    if constexpr (SMALL) {
      scale_m = have > 0 ? e.avg_scale[i / kBlock] : 0.f;
      scale_v = have > 0 ? e.sq_scale[i / kBlock] : 0.f;
    }
  }
  // The step, and its results to where they belong.
  __device__ __forceinline__ void step(const Tensor& e, const StepArgs& a, const StepScalars& s, uint64_t i, int have) const {
    // By itself and not as 1 less it, which has steps of 2^-24 below 1: a rate of 1e-6 times a decay of 0.01 is nothing in them.  The whole change meets the weight in one sum.
    const float fade = float(s.weight_decay * double(e.decay));
    constexpr int kSubnormal = 0x90;   // of either sign
    float xg[N], xp[N], xm[N], xv[N], root[N];
    bool low = false;
    g.widen(xg);
    p.widen(xp);
    if constexpr (SMALL) {
      decode<true>(m, scale_m, xm);
      decode<false>(v, scale_v, xv);
    } else {
      m.widen(xm);
      v.widen(xv);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      {
#pragma clang fp contract(off)
        const float x = xg[k] * s.factor;
        xm[k] = xm[k] * a.beta1 + x * a.beta1c;
        xv[k] = xv[k] * a.beta2 + (x * x) * a.beta2c;
      }
      root[k] = __builtin_amdgcn_sqrtf(xv[k]);
      low |= __builtin_amdgcn_classf(xv[k], kSubnormal);
    }
    if (__builtin_amdgcn_ballot_w64(low) != 0) {   // the machine's root takes them as 0, which would leave m over eps alone
      asm volatile("" ::: "memory");               // stays a branch
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (__builtin_amdgcn_classf(xv[k], kSubnormal)) root[k] = __builtin_amdgcn_sqrtf(xv[k] * 0x1p64f) * 0x1p-32f;
    }
    // eps is 2^-126 or more, so that the reciprocal is finite.  m goes over the root first: where both are tiny that is a number near 1, while m times the rate might lose
    // its bits below 2^-126.
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float away = fmaf(root[k], s.by_second, a.eps);
      xp[k] -= fmaf(xp[k], fade, (xm[k] * __builtin_amdgcn_rcpf(away)) * s.by_first);
    }
    uint32_t bits[N] = {};
    if ((SMALL || KIND == kParamBF16) && a.stochastic) {
      const uint32_t of_tensor = mix(s.of_step + uint32_t(e.ordinal));
#pragma unroll
      for (int k = 0; k < N; ++k) bits[k] = mix(of_tensor + uint32_t(i) + uint32_t(k));
    }
    if constexpr (!SMALL) {
      Numbers<kF32, N>::store_rounded(e.avg, i, have, xm);
      arrived<kOrdered>();
      Numbers<kF32, N>::store_rounded(e.sq, i, have, xv);
      arrived<kOrdered>();
    }
    if constexpr (kMaster) {
      Numbers<kF32, N>::store_rounded(e.master, i, have, xp);
      arrived<kOrdered>();
    }
    if (KIND == kParamBF16 && a.stochastic) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const uint32_t raw = __float_as_uint(xp[k]), up = (raw + (bits[k] * 0x9E3779B1u >> 16)) & 0xffff0000u;
        xp[k] = __uint_as_float(xp[k] == xp[k] ? up : raw);   // the sum leaves infinities what they are, but might carry a NaN beyond
      }
    }
    Numbers<kStored, N>::store_rounded(e.param, i, have, xp);
    if constexpr (SMALL) {
      const float sm = block_scale<true>(xm, kInvTop1), sv = block_scale<false>(xv, kInvTop2);
      first_codes(xm, inverse_of(sm), a.stochastic, bits).store(e.avg, i, have);
      second_codes(xv, root, inverse_of(sv), a.stochastic, bits).store(e.sq, i, have);
      if (i % kBlock == 0 && have > 0) {
        e.avg_scale[i / kBlock] = sm;
        e.sq_scale[i / kBlock] = sv;
      }
    }
  }
};

// Where a workgroup's elements are: chunks hold one unit or several.  The table is read as constant memory, which makes it scalar loads; stores that might
// be to it, for all the compiler knows, would have every pointer read again by vector loads behind them.
struct Place {
  Tensor e;
  uint64_t at;
};
template <class T> using Constant = const __attribute__((address_space(4))) T*;
template <class T> __device__ __forceinline__ T constant_copy(const T* p) {
  struct Raw {
    uint32_t w[sizeof(T) / 4];
  } raw;
  const auto from = (Constant<uint32_t>)reinterpret_cast<uintptr_t>(p);
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 4; ++i) raw.w[i] = from[i];
  return __builtin_bit_cast(T, raw);
}
template <int UNIT> __device__ __forceinline__ Place place_of(const void* table, int32_t count, uint32_t first, uint32_t unit) {
  constexpr uint32_t kUnits = kChunk / UNIT;
  const uint32_t chunk = first + unit / kUnits;
  Place p;
  p.e = constant_copy(tensors_of(table) + constant_copy(map_of(table, count) + chunk));
  p.at = uint64_t(chunk - p.e.first_chunk) * kChunk + unit % kUnits * UNIT;
  return p;
}
// Calls f(element, how many of N the tensor has) for this thread's N elements of a unit; in a unit that is whole, N is a constant.
template <int N, class F> __device__ __forceinline__ void with_elements(const Place& p, F f) {
  const uint64_t i = p.at + threadIdx.x * N;
  if (p.at + kOptNT * N <= uint64_t(p.e.n)) f(i, std::integral_constant<int, N>{});
  else f(i, have_of<N>(p.e.n, i));
}

// A step's scalars: the two powers and quotients by two lanes at once (all of a wave's take part).
__device__ __forceinline__ StepScalars step_scalars(const StepArgs& a) {
  const float factor = a.factor ? a.factor[0] : 1.f;
  const int step = a.step[0];
  const double rate = a.lr * (a.lr_factor ? double(a.lr_factor[0]) : 1.0);
  const bool first = threadIdx.x % 2 == 0;
  double by = first ? a.dbeta1 : a.dbeta2, power = 1.0;   // beta^t for t = step + 1
  for (uint32_t t = uint32_t(step) + 1; t; t >>= 1, by *= by)
    if (t & 1) power *= by;
  const double under = first ? 1.0 - power : sqrt(1.0 - power);
  const int quotient = __float_as_int(float((first ? rate : 1.0) / under));
  return StepScalars{factor, __int_as_float(__builtin_amdgcn_readlane(quotient, 0)), __int_as_float(__builtin_amdgcn_readlane(quotient, 1)),
                     mix(a.seed_lo ^ mix(a.seed_hi ^ mix(uint32_t(step)))), rate * a.weight_decay};
}
// In front of a launch of many workgroups: leaves the scalars in the table and counts the step.
__global__ __launch_bounds__(kWave) void k_step_begin(StepArgs a) {
  const StepScalars s = step_scalars(a);
  if (threadIdx.x != 0) return;
  static_cast<Table*>(a.table)->step = s;
  if (fabsf(s.factor) < INFINITY) a.step[0] += 1;
}

// A workgroup steps four or eight elements a thread and ends: new ones follow in the order of addresses, which the memory serves better than workgroups that walk
// on and drift apart (28 bytes an element in seven streams: 6.3 against 4.3 TB/s), and better still where a wave waits for each access before the next (kOrdered;
// 5.9 without; the 8-bit form is not bound by memory).  ALONE: it works the scalars out itself, and the last workgroup to end counts the step.
template <int KIND, int GRAD, bool SMALL, bool ALONE>
__global__ __launch_bounds__(kOptNT) void k_adamw(StepArgs a) {
  using H = Held<KIND, GRAD, SMALL, ALONE>;
  StepScalars s;
  if constexpr (!ALONE) {
    s = constant_copy<StepScalars>(&static_cast<const Table*>(a.table)->step);
    if (!(fabsf(s.factor) < INFINITY)) return;   // uniform over the launch
  }
  const Place p = place_of<kOptNT * H::N>(a.table, a.count, a.first, a.first_unit + blockIdx.x);
  with_elements<H::N>(p, [&](uint64_t i, int have) {
    H h;
    h.load(p.e, i, have);
    if constexpr (ALONE) s = step_scalars(a);   // while the loads are under way
    if (!ALONE || fabsf(s.factor) < INFINITY) h.step(p.e, a, s, i, have);
  });
  if constexpr (ALONE) {
    if (!(fabsf(s.factor) < INFINITY)) return;
    __syncthreads();   // every wave of this workgroup has read the step by now
    if (threadIdx.x == 0 && count_off(static_cast<Table*>(a.table)->step_tickets)) a.step[0] += 1;
  }
}

using StepKernel = void (*)(StepArgs);
template <int KIND, int GRAD> static StepKernel step_kernel(bool small, bool alone) {
  return small ? (alone ? k_adamw<KIND, GRAD, true, true> : k_adamw<KIND, GRAD, true, false>)
               : (alone ? k_adamw<KIND, GRAD, false, true> : k_adamw<KIND, GRAD, false, false>);
}
template <int KIND> static StepKernel step_kernel(int grad, bool small, bool alone) {
  return grad == 0 ? step_kernel<KIND, kF32>(small, alone) : grad == 1 ? step_kernel<KIND, kBF16>(small, alone) : step_kernel<KIND, kF16>(small, alone);
}
static StepKernel step_kernel(int cls, bool alone) {
  const int kind = cls / 2 / kGrads, grad = cls / 2 % kGrads;
  const bool small = cls % 2;
  switch (kind) {
    case kParamF32: return step_kernel<kParamF32>(grad, small, alone);
    case kParamBF16: return step_kernel<kParamBF16>(grad, small, alone);
    case kMasterBF16: return step_kernel<kMasterBF16>(grad, small, alone);
    default: return step_kernel<kMasterF16>(grad, small, alone);
  }
}
// Up to so many workgroups a step is one launch; of more, working its scalars out and counting off in every one costs more than a launch of its own: one / two
// launches, us, with 32-bit moments 1 M elements 6.7 / 8.6, 4 M 21.5 / 22.6, 17 M 81.0 / 80.4; in 8 bits 1 M 8.6 / 9.3, 4 M 17.6 / 18.1, 8 M 30.4 / 29.8.
constexpr uint32_t kAloneUnits = 4096;

// ---------------------------------------------------------------------------------- moments as numbers
// Bound by bytes: 233 M moments in 8 bits as bf16 220 us (6.4 TB/s).
template <bool SMALL, int DT>
__global__ __launch_bounds__(kOptNT) void k_moments(void* table, int32_t count, uint32_t first, uint32_t first_unit, void* avg, void* sq) {
  constexpr int N = SMALL ? kCodeLane : kWideLane;
  const Place p = place_of<kOptNT * N>(table, count, first, first_unit + blockIdx.x);
  const Tensor& e = p.e;
  with_elements<N>(p, [&](uint64_t i, int have) {
    std::conditional_t<SMALL, Codes, Numbers<kF32, N>> m, v;
    float xm[N], xv[N];
    m.load(e.avg, i, have);
    v.load(e.sq, i, have);
    if constexpr (SMALL) {
      const float scale_m = have > 0 ? e.avg_scale[i / kBlock] : 0.f, scale_v = have > 0 ? e.sq_scale[i / kBlock] : 0.f;
      decode<true>(m, scale_m, xm);
      decode<false>(v, scale_v, xv);
    } else {
      m.widen(xm);
      v.widen(xv);
    }
    Numbers<DT, N>::store_rounded(avg, uint64_t(e.out) + i, have, xm);
    Numbers<DT, N>::store_rounded(sq, uint64_t(e.out) + i, have, xv);
  });
}

// ---------------------------------------------------------------------------------- norm
// Workgroups, and up to how many chunks a launch does it all: one / two launches, us, 200 tensors of 30 K elements in all 4.1 / 6.3, 1 M bf16 4.5 / 6.4, 2 M 5.7 / 6.3, 3 M
// 6.3 / 6.2.
constexpr int kNormMax = 2048, kNormAlone = 1024;
template <int DT> __device__ __forceinline__ double squares(const Place& p) {
  double sum = 0.0;
  with_elements<kCodeLane>(p, [&](uint64_t i, int have) {
    Numbers<DT, kCodeLane> g;
    float x[kCodeLane];
    g.load(p.e.grad, i, have);
    g.widen(x);
#pragma unroll
    for (int k = 0; k < kCodeLane; ++k) sum = fma(double(x[k]), double(x[k]), sum);
  });
  return sum;
}
struct NormOut {
  float grad_scale, max_norm;
  float *norm, *factor;
};
__device__ __forceinline__ double workgroup_sum(double sum, double* lds /*[kOptNT / kWave]*/) {   // in thread 0
  sum = wave_sum_d(sum);
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < kOptNT / kWave; ++w) sum += lds[w];
  return sum;
}
__device__ __forceinline__ void norm_out(const NormOut& o, double sum) {
  const double x = fabs(double(o.grad_scale)) * sqrt(sum);
  if (o.norm) o.norm[0] = float(x);
  if (!o.factor) return;
  double f = double(o.grad_scale);
  if (!(sum < INFINITY)) f = __builtin_nan("");
  else if (o.max_norm > 0.f && x > double(o.max_norm)) f *= double(o.max_norm) / x;
  o.factor[0] = float(f);
}
// ALONE: the last workgroup to end adds up the others' parts.  They are written and read where all compute units see the same, and a part is there before its
// workgroup counts itself, so that no cache has to be written back for it.
template <bool ALONE>
__global__ __launch_bounds__(kOptNT) void k_norm_parts(void* table, int32_t count, uint32_t chunks, double* part, NormOut out) {
  __shared__ double lds[2][kOptNT / kWave];
  __shared__ bool last;
  double sum = 0.0;
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Place p = place_of<kChunk>(table, count, 0, c);
    const int grad = p.e.kind / 2 % kGrads;
    sum += grad == 0 ? squares<kF32>(p) : grad == 1 ? squares<kBF16>(p) : squares<kF16>(p);
  }
  sum = workgroup_sum(sum, lds[0]);
  if constexpr (!ALONE) {
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
  } else {
    if (threadIdx.x == 0) {
      __hip_atomic_store(&part[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      arrived<true>();
      last = count_off(static_cast<Table*>(table)->norm_tickets);
    }
    __syncthreads();
    if (!last) return;
    sum = 0.0;
    for (uint32_t k = threadIdx.x; k < gridDim.x; k += kOptNT) sum += __hip_atomic_load(&part[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = workgroup_sum(sum, lds[1]);
    if (threadIdx.x == 0) norm_out(out, sum);
  }
}
__global__ __launch_bounds__(kOptNT) void k_norm_end(const double* __restrict__ part, int n, NormOut out) {
  __shared__ double lds[kOptNT / kWave];
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kOptNT) sum += part[k];
  sum = workgroup_sum(sum, lds);
  if (threadIdx.x == 0) norm_out(out, sum);
}

// Launches over the classes that have parameters, a workgroup to a unit: launch(class, its first unit, how many).
constexpr int kFirstClass = class_of(kParamF32, 0, 0);
constexpr uint32_t kMostUnits = (1u << 24) - 1;   // workgroups of 256 threads that a launch has at most
static uint64_t units_of(const Table* t, int k) {
  return uint64_t(t->class_first[k + 1] - t->class_first[k]) * (kChunk / (kOptNT * (k % 2 ? kCodeLane : kWideLane)));
}
template <class Launch> static void for_classes(const Table* t, Launch launch) {
  for (int k = kFirstClass; k < kClasses; ++k) {
    const uint64_t units = units_of(t, k);
    for (uint64_t from = 0; from < units; from += kMostUnits) launch(k, uint32_t(from), unsigned(units - from < kMostUnits ? units - from : kMostUnits));
  }
}

size_t grad_norm_workspace_bytes() { return kNormMax * sizeof(double); }

// Workgroups of a launch over so many chunks: as many as are under way at once, each of which walks on.
static unsigned opt_grid(uint32_t chunks, int per_cu) {
  const uint32_t most = uint32_t(compute_units()) * per_cu;
  return chunks < most ? chunks : most;
}

}  // namespace aero

extern "C" size_t aero_tensor_table_bytes(const aero_tensor* list, int32_t count) {
  if (count < 0 || (count > 0 && !list)) return 0;
  uint64_t chunks = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (list[k].n < 0) return 0;
    chunks += aero::chunks_of(list[k]);
  }
  return (aero::map_offset(count) + size_t(chunks) * 4 + 15) / 16 * 16;
}

extern "C" aero_status aero_tensor_table(const aero_tensor* list, int32_t count, void* image, size_t image_bytes) {
  using namespace aero;
  if (count < 0 || count >= (1 << 20)) return AERO_ERR_SHAPE;
  if ((count > 0 && !list) || !image) return AERO_ERR_NULL;
  uint64_t chunks = 0, of_class[kClasses] = {};
  for (int32_t k = 0; k < count; ++k) {
    const aero_status st = check_tensor(list[k]);
    if (st != AERO_OK) return st;
    chunks += chunks_of(list[k]);
    of_class[class_of(list[k])] += chunks_of(list[k]);
  }
  if (chunks >= (uint64_t(1) << 30)) return AERO_ERR_SHAPE;   // units of half a chunk count in 32 bits
  const size_t bytes = aero_tensor_table_bytes(list, count);
  if (image_bytes < bytes) return AERO_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(image) % 16 != 0) return AERO_ERR_ALIGN;
  std::memset(image, 0, bytes);
  Table* t = static_cast<Table*>(image);
  t->magic = kMagic;
  t->bytes = bytes;
  t->count = count;
  t->chunks = uint32_t(chunks);
  uint32_t next[kClasses];
  for (int k = 0; k < kClasses; ++k) {
    next[k] = t->class_first[k];
    t->class_first[k + 1] = t->class_first[k] + uint32_t(of_class[k]);
  }
  Tensor* tensors = const_cast<Tensor*>(tensors_of(image));
  uint32_t* map = const_cast<uint32_t*>(map_of(image, count));
  int64_t out = 0;
  for (int32_t k = 0; k < count; ++k) {
    const aero_tensor& x = list[k];
    const int cls = class_of(x);
    const uint32_t n = uint32_t(chunks_of(x));
    tensors[k] = Tensor{static_cast<char*>(x.param), static_cast<const char*>(x.grad), x.master, static_cast<char*>(x.exp_avg),
                        static_cast<char*>(x.exp_avg_sq), x.exp_avg_scale, x.exp_avg_sq_scale, x.n, out, next[cls], k, x.decay, cls};
    for (uint32_t c = 0; c < n; ++c) map[next[cls] + c] = uint32_t(k);
    next[cls] += n;
    if (x.param) out += x.n;
  }
  return AERO_OK;
}

extern "C" aero_status aero_grad_norm(const void* image, void* table, float grad_scale, float max_norm, float* norm, float* factor,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (!image || !table) return AERO_ERR_NULL;
  const Table* t = table_of(image);
  if (!t || !(grad_scale - grad_scale == 0.f) || max_norm != max_norm) return AERO_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(table) % 16 != 0) return AERO_ERR_ALIGN;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < grad_norm_workspace_bytes()) return AERO_ERR_WORKSPACE;
  double* part = static_cast<double*>(workspace);
  hipStream_t s = as_stream(stream);
  const NormOut out{grad_scale, max_norm, norm, factor};
  if (t->chunks > 0 && t->chunks <= uint32_t(kNormAlone)) {
    hipLaunchKernelGGL(k_norm_parts<true>, dim3(t->chunks), dim3(kOptNT), 0, s, table, t->count, t->chunks, part, out);
    return launch_status();
  }
  unsigned grid = opt_grid(t->chunks, 8);
  if (grid > unsigned(kNormMax)) grid = kNormMax;
  if (grid > 0) hipLaunchKernelGGL(k_norm_parts<false>, dim3(grid), dim3(kOptNT), 0, s, table, t->count, t->chunks, part, out);
  hipLaunchKernelGGL(k_norm_end, dim3(1), dim3(kOptNT), 0, s, part, int(grid), out);
  return launch_status();
}

extern "C" aero_status aero_adamw_step(const void* image, void* table, const aero_adamw_params* p, int32_t* step, const float* factor,
                                       const float* lr_factor, void* stream) {
  using namespace aero;
  if (!image || !table || !p || !step) return AERO_ERR_NULL;
  const Table* t = table_of(image);
  if (!t) return AERO_ERR_SHAPE;
  if (!(p->beta1 >= 0.0 && p->beta1 < 1.0 && p->beta2 >= 0.0 && p->beta2 < 1.0)) return AERO_ERR_SHAPE;
  if (!(float(p->eps) >= 0x1p-126f) || !std::isfinite(float(p->eps)) || !(p->lr >= 0.0) || !std::isfinite(p->lr) || !std::isfinite(p->weight_decay))
    return AERO_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(table) % 16 != 0) return AERO_ERR_ALIGN;
  hipStream_t s = as_stream(stream);
  StepArgs a{};
  a.table = table;
  a.count = t->count;
  a.beta1 = float(p->beta1);
  a.beta1c = float(1.0 - p->beta1);
  a.beta2 = float(p->beta2);
  a.beta2c = float(1.0 - p->beta2);
  a.eps = float(p->eps);
  a.lr = p->lr;
  a.weight_decay = p->weight_decay;
  a.dbeta1 = p->beta1;
  a.dbeta2 = p->beta2;
  a.seed_lo = uint32_t(p->seed);
  a.seed_hi = uint32_t(p->seed >> 32);
  a.stochastic = p->stochastic != 0;
  a.step = step;
  a.factor = factor;
  a.lr_factor = lr_factor;
  int classes = 0, only = 0;
  for (int k = kFirstClass; k < kClasses; ++k) {
    if (t->class_first[k + 1] > t->class_first[k]) {
      ++classes;
      only = k;
    }
  }
  const uint64_t alone = classes == 1 ? units_of(t, only) : 0;
  if (alone > 0 && alone <= kAloneUnits) {
    a.first = t->class_first[only];
    hipLaunchKernelGGL(step_kernel(only, true), dim3(unsigned(alone)), dim3(kOptNT), 0, s, a);
    return launch_status();
  }
  hipLaunchKernelGGL(k_step_begin, dim3(1), dim3(kWave), 0, s, a);
  for_classes(t, [&](int k, uint32_t first_unit, unsigned n) {
    a.first = t->class_first[k];
    a.first_unit = first_unit;
    hipLaunchKernelGGL(step_kernel(k, false), dim3(n), dim3(kOptNT), 0, s, a);
  });
  return launch_status();
}

extern "C" aero_status aero_adamw_moments(const void* image, void* table, int32_t dtype, void* avg, void* avg_sq, void* stream) {
  using namespace aero;
  if (!image || !table) return AERO_ERR_NULL;
  const Table* t = table_of(image);
  if (!t) return AERO_ERR_SHAPE;
  if (dtype != AERO_F32 && dtype != AERO_BF16) return AERO_ERR_DTYPE;
  if (t->chunks == t->class_first[kFirstClass]) return AERO_OK;
  if (!avg || !avg_sq) return AERO_ERR_NULL;
  const uintptr_t both = reinterpret_cast<uintptr_t>(avg) | reinterpret_cast<uintptr_t>(avg_sq);
  if (both % storage_bytes(dtype) != 0 || reinterpret_cast<uintptr_t>(table) % 16 != 0) return AERO_ERR_ALIGN;
  hipStream_t s = as_stream(stream);
  for_classes(t, [&](int k, uint32_t first_unit, unsigned n) {
    const auto kernel = k % 2 ? (dtype == AERO_F32 ? k_moments<true, kF32> : k_moments<true, kBF16>)
                              : (dtype == AERO_F32 ? k_moments<false, kF32> : k_moments<false, kBF16>);
    hipLaunchKernelGGL(kernel, dim3(n), dim3(kOptNT), 0, s, table, t->count, t->class_first[k], first_unit, avg, avg_sq);
  });
  return launch_status();
}
