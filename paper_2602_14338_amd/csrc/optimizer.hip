// What happens to gradients: their norm over many tensors, and Adam's step with decoupled weight decay on all of them at once, with moments
// in 32 bits or in 8.
//
// A table describes the tensors.  Its elements are dealt out in chunks of 2048 of one tensor, 8 to a thread; the chunks of tensors of one class
// (types of parameter, gradient and moments) stand together, and a class is one launch.
//
// Both are bound by bytes: n of the gradient, and for a step what is read and written of weights and moments, 28 bytes an element for
// 16-bit weights with a master and 32-bit moments, 10 for 16-bit weights with 8-bit moments.
#include <cmath>
#include <cstring>

#include "row_scan.h"

namespace aero {

// ---------------------------------------------------------------------------------- the table
constexpr int kOptNT = 256, kPer = 4, kBlock = AERO_MOMENT_BLOCK, kUnit = kBlock * (kOptNT / kWave), kUnits = 2, kChunk = kUnit * kUnits;
static_assert(kBlock == kWave * kPer, "a wave holds a block of moments");

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

constexpr uint64_t kMagic = 0x41455254'61626c65ull;
struct Table {
  uint64_t magic;
  uint64_t bytes;
  int32_t count;
  uint32_t chunks;
  uint32_t ticket;        // of the step's workgroups (device copy)
  uint32_t pad;
  StepScalars step;       // of the step under way (device copy)
  uint32_t class_first[kClasses + 1];   // chunks of class k: class_first[k] .. class_first[k + 1]
  uint32_t pad2[3];
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
// A thread's elements come in groups of four, the groups of a wave's lanes side by side: 64 lanes read and write 256 elements in a row.  Any
// alignment, and past the caches: nothing is read twice.
typedef uint32_t u32_any_t __attribute__((aligned(1)));
// Waits for what this wave has under way in memory, if asked to.
template <bool ASKED> __device__ __forceinline__ void arrived() {
  if constexpr (ASKED) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    asm volatile("" ::: "memory");
  }
}
// How many of the four elements from i on a tensor of n has.
__device__ __forceinline__ int have_of(int64_t n, uint64_t i) {
  const int64_t behind = n - int64_t(i);
  return behind >= kPer ? kPer : behind > 0 ? int(behind) : 0;
}
// Four stored elements: `have` of them are the tensor's, the others read as 0 and are not written.
template <int DT> struct Four {
  static constexpr bool kWide = DT == kF32;
  using raw = std::conditional_t<kWide, f32x4_any_t, u32x2_any_t>;
  __device__ __forceinline__ static raw load(const void* base, uint64_t i, int have) {
    const char* p = static_cast<const char*>(base) + i * Storage<DT>::kBytes;
    if (have >= kPer) return __builtin_nontemporal_load(reinterpret_cast<const raw*>(p));
    if constexpr (kWide) {
      const float* f = reinterpret_cast<const float*>(p);
      return raw{have > 0 ? f[0] : 0.f, have > 1 ? f[1] : 0.f, have > 2 ? f[2] : 0.f, 0.f};
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
      return raw{(have > 0 ? uint32_t(h[0]) : 0u) | (have > 1 ? uint32_t(h[1]) << 16 : 0u), have > 2 ? uint32_t(h[2]) : 0u};
    }
  }
  __device__ __forceinline__ static void widen(const raw& a, float (&x)[kPer]) {
    if constexpr (kWide) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = a[k];
    } else if constexpr (DT == kBF16) {
      x[0] = bf16_lo(a.x), x[1] = bf16_hi(a.x), x[2] = bf16_lo(a.y), x[3] = bf16_hi(a.y);
    } else {
      x[0] = f16_to_f32(uint16_t(a.x)), x[1] = f16_to_f32(uint16_t(a.x >> 16));
      x[2] = f16_to_f32(uint16_t(a.y)), x[3] = f16_to_f32(uint16_t(a.y >> 16));
    }
  }
  __device__ __forceinline__ static void store(void* base, uint64_t i, int have, const float (&x)[kPer]) {
    char* p = static_cast<char*>(base) + i * Storage<DT>::kBytes;
    if (have < kPer) {
#pragma unroll
      for (int k = 0; k < kPer - 1; ++k)
        if (k < have) store_elt<DT>(p, k, x[k]);
      return;
    }
    if constexpr (kWide) {
      __builtin_nontemporal_store((raw{x[0], x[1], x[2], x[3]}), reinterpret_cast<raw*>(p));
    } else {
      const auto pack = [](float lo, float hi) { return DT == kBF16 ? pack_bf16x2(lo, hi) : pack_f16x2(lo, hi); };
      __builtin_nontemporal_store((raw{pack(x[0], x[1]), pack(x[2], x[3])}), reinterpret_cast<raw*>(p));
    }
  }
};
__device__ __forceinline__ uint32_t load_codes(const char* base, uint64_t i, int have) {
  if (have >= kPer) return __builtin_nontemporal_load(reinterpret_cast<const u32_any_t*>(base + i));
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (k < have) w |= uint32_t(uint8_t(base[i + k])) << (8 * k);
  return w;
}
__device__ __forceinline__ void store_codes(char* base, uint64_t i, int have, uint32_t w) {
  if (have >= kPer) {
    __builtin_nontemporal_store(w, reinterpret_cast<u32_any_t*>(base + i));
    return;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (k < have) base[i + k] = char(w >> (8 * k));
}

// ---------------------------------------------------------------------------------- moments in 8 bits
// Codes and values as aero.h defines them; each product, sum and quotient rounded by itself (no fused multiply-add), so that the codes are a
// function of the definition alone.
constexpr float kTop1 = 16129.f, kTop2 = 4228250625.f;   // 127^2, 255^4
constexpr float kInvTop1 = float(1.0 / 16129.0), kInvTop2 = float(1.0 / 4228250625.0);
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
template <bool FIRST> __device__ __forceinline__ void decode4(uint32_t w, float scale, float (&x)[kPer]) {
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if constexpr (FIRST) x[k] = first_value(float(int8_t(w >> (8 * k))), scale);
    else x[k] = second_value(float(w >> (8 * k) & 0xff), scale);
  }
}
// The scale of a block, four of whose moments each lane of a wave holds.  The largest by its bits: as whole numbers infinities and NaN come out largest.
template <bool SIGNED> __device__ __forceinline__ float block_scale(const float (&x)[kPer], float inv_top) {
#pragma clang fp contract(off)
  auto most = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  auto bits = [](float v) { return SIGNED ? __float_as_uint(v) & 0x7fffffffu : __float_as_uint(v); };
  uint32_t m = most(most(bits(x[0]), bits(x[1])), most(bits(x[2]), bits(x[3])));
  m = uint32_t(wave_reduce_i(int(m), [&](int a, int b) { return int(most(uint32_t(a), uint32_t(b))); }));
  if (m >= 0x7f800000u) return __builtin_nanf("");
  const float s = __uint_as_float(m) * inv_top;
  return s >= 1.17549435e-38f ? s : 0.f;
}
// Codes of a block's moments, of which this lane has four.  The root that finds a code is an estimate from below, by more than its own error and by so little that
// the next code is rarely the right one: a branch that few waves take.
constexpr float kBelow = 1.f - 0x1p-21f;
__device__ __forceinline__ uint32_t first_codes(const float (&x)[kPer], float inv, const float (&u)[kPer]) {
#pragma clang fp contract(off)
  float y[kPer], c[kPer];
  bool more = false;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    y[k] = fminf(fabsf(x[k]) * inv, kTop1);
    c[k] = floorf(__builtin_amdgcn_sqrtf(y[k]) * kBelow);
    const float next = c[k] + 1.f;
    more |= next * next <= y[k];
  }
  if (__builtin_amdgcn_ballot_w64(more) != 0) {
    asm volatile("" ::: "memory");   // stays a branch
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const float next = c[k] + 1.f;
      if (next * next <= y[k]) c[k] = next;
    }
  }
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (u[k] * (2.f * c[k] + 1.f) < y[k] - c[k] * c[k]) c[k] += 1.f;
    w |= (uint32_t(int(x[k] < 0.f ? -c[k] : c[k])) & 0xff) << (8 * k);
  }
  return w;
}
__device__ __forceinline__ uint32_t second_codes(const float (&x)[kPer], float inv, const float (&u)[kPer]) {
#pragma clang fp contract(off)
  float y[kPer], c[kPer], at[kPer], next[kPer];
  bool more = false;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    y[k] = fminf(x[k] * inv, kTop2);
    c[k] = floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(y[k])) * kBelow);
    at[k] = fourth(c[k]);
    next[k] = fourth(c[k] + 1.f);
    more |= next[k] <= y[k];
  }
  if (__builtin_amdgcn_ballot_w64(more) != 0) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (next[k] <= y[k]) {
        c[k] += 1.f;
        at[k] = next[k];
        next[k] = fourth(c[k] + 1.f);
      }
    }
  }
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (u[k] * (next[k] - at[k]) < y[k] - at[k]) c[k] += 1.f;
    const float least = y[k] > 0.f ? 1.f : 0.f;   // a moment > 0 is not stored as 0
    w |= uint32_t(__builtin_amdgcn_fmed3f(c[k], least, 255.f)) << (8 * k);
  }
  return w;
}

__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}
__device__ __forceinline__ float uniform16(uint32_t low16) { return fmaf(float(low16), 0x1p-16f, 0x1p-17f); }   // exact

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

// b^t for a whole t >= 1.
__device__ __forceinline__ double power(double b, uint32_t t) {
  double r = 1.0;
  for (; t; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// What a lane has of an element group, as it is stored: to be widened when it is worked on, so that the loads of a group are under way together, and those of
// the next one while this one is stepped.
template <int KIND, int GRAD, bool SMALL, bool ALONE> struct Held {
  static constexpr bool kOrdered = !SMALL && !ALONE;
  static constexpr bool kMaster = KIND == kMasterBF16 || KIND == kMasterF16;
  static constexpr int kStored = KIND == kParamF32 ? kF32 : KIND == kMasterF16 ? kF16 : kBF16, kRead = kMaster ? kF32 : kStored;
  typename Four<GRAD>::raw g;
  typename Four<kRead>::raw p;
  Four<kF32>::raw m, v;       // 32-bit moments
  uint32_t wm, wv;            // codes
  float scale_m, scale_v;

  __device__ __forceinline__ void load(const Tensor& e, uint64_t from, int lane, int have) {
    const uint64_t i = from + lane * kPer;
    g = Four<GRAD>::load(e.grad, i, have);
    arrived<kOrdered>();
    if constexpr (kMaster) p = Four<kF32>::load(e.master, i, have);
    else p = Four<kRead>::load(e.param, i, have);
    arrived<kOrdered>();
    if constexpr (SMALL) {
      wm = load_codes(e.avg, i, have);
      wv = load_codes(e.sq, i, have);
      const bool in = from < uint64_t(e.n);
      scale_m = in ? e.avg_scale[from / kBlock] : 0.f;
      scale_v = in ? e.sq_scale[from / kBlock] : 0.f;
    } else {
      m = Four<kF32>::load(e.avg, i, have);
      arrived<kOrdered>();
      v = Four<kF32>::load(e.sq, i, have);
    }
  }
  // The step of the group, and its results to where they belong.
  __device__ __forceinline__ void step(const Tensor& e, const StepArgs& a, const StepScalars& s, uint64_t from, int lane, int have) const {
    const uint64_t i = from + lane * kPer;
    const float keep = float(s.weight_decay);
    const uint32_t of_tensor = mix(s.of_step + uint32_t(e.ordinal));
    float xg[kPer], xp[kPer], xm[kPer], xv[kPer];
    Four<GRAD>::widen(g, xg);
    Four<kRead>::widen(p, xp);
    if constexpr (SMALL) {
      decode4<true>(wm, scale_m, xm);
      decode4<false>(wv, scale_v, xv);
    } else {
      Four<kF32>::widen(m, xm);
      Four<kF32>::widen(v, xv);
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      {
#pragma clang fp contract(off)
        const float x = xg[k] * s.factor;
        xm[k] = xm[k] * a.beta1 + x * a.beta1c;
        xv[k] = xv[k] * a.beta2 + (x * x) * a.beta2c;
      }
      const float away = fmaf(__builtin_amdgcn_sqrtf(xv[k]), s.by_second, a.eps);
      xp[k] = fmaf(xp[k], keep, -(xm[k] * s.by_first) * __builtin_amdgcn_rcpf(away));
    }
    uint32_t bits[kPer];
    if ((SMALL || KIND == kParamBF16) && a.stochastic) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) bits[k] = mix(of_tensor + uint32_t(i) + uint32_t(k));
    }
    if constexpr (!SMALL) {
      Four<kF32>::store(e.avg, i, have, xm);
      arrived<kOrdered>();
      Four<kF32>::store(e.sq, i, have, xv);
      arrived<kOrdered>();
    }
    if constexpr (kMaster) {
      Four<kF32>::store(e.master, i, have, xp);
      arrived<kOrdered>();
    }
    if (KIND == kParamBF16 && a.stochastic) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const uint32_t raw = __float_as_uint(xp[k]), up = (raw + (bits[k] * 0x9E3779B1u >> 16)) & 0xffff0000u;
        xp[k] = __uint_as_float(fabsf(xp[k]) < INFINITY ? up : raw);
      }
    }
    Four<kStored>::store(e.param, i, have, xp);
    if constexpr (SMALL) {
      const float sm = block_scale<true>(xm, kInvTop1), sv = block_scale<false>(xv, kInvTop2);
      const float im = sm > 0.f ? 1.f / sm : 0.f, iv = sv > 0.f ? 1.f / sv : 0.f;
      float um[kPer], uv[kPer];
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        um[k] = a.stochastic ? uniform16(bits[k] & 0xffff) : 0.5f;
        uv[k] = a.stochastic ? uniform16(bits[k] >> 16) : 0.5f;
      }
      store_codes(e.avg, i, have, first_codes(xm, im, um));
      store_codes(e.sq, i, have, second_codes(xv, iv, uv));
      if (lane == 0 && have > 0) {
        e.avg_scale[from / kBlock] = sm;
        e.sq_scale[from / kBlock] = sv;
      }
    }
  }
};

// Where a wave's group of a unit is: units are the halves, quarters, ... of chunks that a workgroup takes at a time.  The table is read as constant memory, which
// makes it scalar loads; stores that might be to it, for all the compiler knows, would have every pointer read again by vector loads behind them.
struct Place {
  Tensor e;
  uint64_t from;
  bool full;   // the tensor has all of the workgroup's unit
};
template <class T> using Constant = const __attribute__((address_space(4))) T*;
template <class T> __device__ __forceinline__ T constant_copy(const T* p) {
  struct Words {
    uint32_t w[sizeof(T) / 4];
  } words;
  const auto from = (Constant<uint32_t>)reinterpret_cast<uintptr_t>(p);
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 4; ++i) words.w[i] = from[i];
  return __builtin_bit_cast(T, words);
}
__device__ __forceinline__ Place place_of(const void* table, int32_t count, uint32_t first, uint32_t unit, int wave) {
  const uint32_t chunk = first + unit / kUnits;
  Place p;
  p.e = constant_copy(tensors_of(table) + constant_copy(map_of(table, count) + chunk));
  const uint64_t at = uint64_t(chunk - p.e.first_chunk) * kChunk + unit % kUnits * kUnit;
  p.from = at + uint64_t(wave) * kBlock;
  p.full = at + kUnit <= uint64_t(p.e.n);
  return p;
}

// Works out a step's scalars, counts it, and leaves them in the table for a launch of many workgroups.
__device__ __forceinline__ StepScalars step_scalars(const StepArgs& a, float factor, int step) {
  const uint32_t t = uint32_t(step) + 1;
  const double rate = a.lr * (a.lr_factor ? double(a.lr_factor[0]) : 1.0);
  return StepScalars{factor, float(rate / (1.0 - power(a.dbeta1, t))), float(1.0 / sqrt(1.0 - power(a.dbeta2, t))),
                     mix(a.seed_lo ^ mix(a.seed_hi ^ mix(uint32_t(step)))), rate * a.weight_decay};
}
__global__ void k_step_begin(StepArgs a) {
  const float factor = a.factor ? a.factor[0] : 1.f;
  static_cast<Table*>(a.table)->step = step_scalars(a, factor, a.step[0]);
  if (fabsf(factor) < INFINITY) a.step[0] += 1;
}

// A workgroup steps 1024 elements and ends.  ALONE: it works the scalars out itself, and the last workgroup to end counts the step.
template <int KIND, int GRAD, bool SMALL, bool ALONE>
__global__ __launch_bounds__(kOptNT) void k_adamw(StepArgs a) {
  int step = 0;
  StepScalars s;
  if constexpr (ALONE) {
    step = a.step[0];
    s = step_scalars(a, a.factor ? a.factor[0] : 1.f, step);
  } else {
    s = constant_copy<StepScalars>(&static_cast<const Table*>(a.table)->step);
  }
  if (!(fabsf(s.factor) < INFINITY)) return;   // uniform over the launch
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Place p = place_of(a.table, a.count, a.first, a.first_unit + blockIdx.x, wave);
  s.weight_decay = 1.0 - s.weight_decay * double(p.e.decay);
  Held<KIND, GRAD, SMALL, ALONE> h;
  if (p.full) {
    h.load(p.e, p.from, lane, kPer);
    h.step(p.e, a, s, p.from, lane, kPer);
  } else {
    const int have = have_of(p.e.n, p.from + lane * kPer);
    h.load(p.e, p.from, lane, have);
    h.step(p.e, a, s, p.from, lane, have);
  }
  if constexpr (ALONE) {
    __syncthreads();   // every wave of this workgroup has read the step by now
    if (threadIdx.x == 0) {
      uint32_t* ticket = &static_cast<Table*>(a.table)->ticket;
      if (atomicAdd(ticket, 1u) == gridDim.x - 1) {
        *ticket = 0;
        a.step[0] = step + 1;
      }
    }
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
// Up to so many workgroups a step is one launch; of more, working its scalars out and counting off in every one would cost more than a launch of its own.
constexpr uint32_t kAloneUnits = 1024;

// ---------------------------------------------------------------------------------- moments as numbers
template <bool SMALL> struct HeldMoments {
  Four<kF32>::raw m, v;
  uint32_t wm, wv;
  float scale_m, scale_v;
  __device__ __forceinline__ void load(const Tensor& e, uint64_t from, int lane, int have) {
    const uint64_t i = from + lane * kPer;
    if constexpr (SMALL) {
      wm = load_codes(e.avg, i, have);
      wv = load_codes(e.sq, i, have);
      const bool in = from < uint64_t(e.n);
      scale_m = in ? e.avg_scale[from / kBlock] : 0.f;
      scale_v = in ? e.sq_scale[from / kBlock] : 0.f;
    } else {
      m = Four<kF32>::load(e.avg, i, have);
      v = Four<kF32>::load(e.sq, i, have);
    }
  }
  template <int DT> __device__ __forceinline__ void store(void* avg, void* sq, uint64_t i, int have) const {
    float xm[kPer], xv[kPer];
    if constexpr (SMALL) {
      decode4<true>(wm, scale_m, xm);
      decode4<false>(wv, scale_v, xv);
    } else {
      Four<kF32>::widen(m, xm);
      Four<kF32>::widen(v, xv);
    }
    Four<DT>::store(avg, i, have, xm);
    Four<DT>::store(sq, i, have, xv);
  }
};
template <bool SMALL, int DT>
__global__ __launch_bounds__(kOptNT) void k_moments(void* table, int32_t count, uint32_t first, void* avg, void* sq) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  {
    HeldMoments<SMALL> h[kUnits];
    const Place p = place_of(table, count, first, blockIdx.x * kUnits, wave);
    const bool full = p.from - uint64_t(wave) * kBlock + kChunk <= uint64_t(p.e.n);
    const auto all = [&](auto have) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u) h[u].load(p.e, p.from + u * kUnit, lane, have(p.from + u * kUnit + lane * kPer));
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        h[u].template store<DT>(avg, sq, uint64_t(p.e.out) + p.from + u * kUnit + lane * kPer, have(p.from + u * kUnit + lane * kPer));
    };
    if (full) all([](uint64_t) { return kPer; });
    else all([&](uint64_t i) { return have_of(p.e.n, i); });
  }
}

// ---------------------------------------------------------------------------------- norm
constexpr int kNormMax = 2048;   // workgroups
template <int DT, class Have> __device__ __forceinline__ void add_squares(const Place& p, int lane, Have have, double& sum) {
  typename Four<DT>::raw g[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const uint64_t i = p.from + u * kUnit + lane * kPer;
    g[u] = Four<DT>::load(p.e.grad, i, have(i));
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    float x[kPer];
    Four<DT>::widen(g[u], x);
#pragma unroll
    for (int k = 0; k < kPer; ++k) sum = fma(double(x[k]), double(x[k]), sum);
  }
}
__global__ __launch_bounds__(kOptNT) void k_norm_parts(const void* table, int32_t count, uint32_t chunks, double* __restrict__ part) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  double sum = 0.0;
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Place p = place_of(table, count, 0, c * kUnits, wave);
    const bool full = p.from - uint64_t(wave) * kBlock + kChunk <= uint64_t(p.e.n);
    const int grad = p.e.kind / 2 % kGrads;
    const auto add = [&](auto have) {
      if (grad == 0) add_squares<kF32>(p, lane, have, sum);
      else if (grad == 1) add_squares<kBF16>(p, lane, have, sum);
      else add_squares<kF16>(p, lane, have, sum);
    };
    if (full) add([](uint64_t) { return kPer; });
    else add([&](uint64_t i) { return have_of(p.e.n, i); });
  }
  sum = wave_sum_d(sum);
  __shared__ double s_sum[kOptNT / kWave];
  if (threadIdx.x % kWave == 0) s_sum[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kOptNT / kWave; ++w) sum += s_sum[w];
    part[blockIdx.x] = sum;
  }
}
__global__ __launch_bounds__(kOptNT) void k_norm_end(const double* __restrict__ part, int n, float grad_scale, float max_norm,
                                                     float* __restrict__ norm, float* __restrict__ factor) {
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kOptNT) sum += part[k];
  sum = wave_sum_d(sum);
  __shared__ double s_sum[kOptNT / kWave];
  if (threadIdx.x % kWave == 0) s_sum[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kOptNT / kWave; ++w) sum += s_sum[w];
  const double x = fabs(double(grad_scale)) * sqrt(sum);
  if (norm) norm[0] = float(x);
  if (!factor) return;
  double f = double(grad_scale);
  if (!(sum < INFINITY)) f = __builtin_nan("");
  else if (max_norm > 0.f && x > double(max_norm)) f *= double(max_norm) / x;
  factor[0] = float(f);
}

constexpr uint32_t kMostUnits = (1u << 24) - 1;   // workgroups of 256 threads that a launch has at most

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
  if (chunks * kUnits >= (uint64_t(1) << 31)) return AERO_ERR_SHAPE;
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
  unsigned grid = opt_grid(t->chunks, 8);
  if (grid > unsigned(kNormMax)) grid = kNormMax;
  if (grid > 0) hipLaunchKernelGGL(k_norm_parts, dim3(grid), dim3(kOptNT), 0, s, table, t->count, t->chunks, part);
  hipLaunchKernelGGL(k_norm_end, dim3(1), dim3(kOptNT), 0, s, part, int(grid), grad_scale, max_norm, norm, factor);
  return launch_status();
}

extern "C" aero_status aero_adamw_step(const void* image, void* table, const aero_adamw_params* p, int32_t* step, const float* factor,
                                       const float* lr_factor, void* stream) {
  using namespace aero;
  if (!image || !table || !p || !step) return AERO_ERR_NULL;
  const Table* t = table_of(image);
  if (!t) return AERO_ERR_SHAPE;
  if (!(p->beta1 >= 0.0 && p->beta1 < 1.0 && p->beta2 >= 0.0 && p->beta2 < 1.0)) return AERO_ERR_SHAPE;
  if (!(float(p->eps) > 0.f) || !std::isfinite(float(p->eps)) || !(p->lr >= 0.0) || !std::isfinite(p->lr) || !std::isfinite(p->weight_decay))
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
  constexpr int kFirst = class_of(kParamF32, 0, 0);
  int classes = 0, only = 0;
  for (int k = kFirst; k < kClasses; ++k) {
    if (t->class_first[k + 1] > t->class_first[k]) {
      ++classes;
      only = k;
    }
  }
  const uint64_t units = uint64_t(t->class_first[kClasses] - t->class_first[kFirst]) * kUnits;
  if (classes == 1 && units <= kAloneUnits) {
    a.first = t->class_first[only];
    hipLaunchKernelGGL(step_kernel(only, true), dim3(unsigned(units)), dim3(kOptNT), 0, s, a);
    return launch_status();
  }
  hipLaunchKernelGGL(k_step_begin, dim3(1), dim3(1), 0, s, a);
  for (int k = kFirst; k < kClasses; ++k) {
    const uint64_t of_class = uint64_t(t->class_first[k + 1] - t->class_first[k]) * kUnits;
    a.first = t->class_first[k];
    for (uint64_t from = 0; from < of_class; from += kMostUnits) {
      const uint64_t n = of_class - from < kMostUnits ? of_class - from : kMostUnits;
      a.first_unit = uint32_t(from);
      hipLaunchKernelGGL(step_kernel(k, false), dim3(unsigned(n)), dim3(kOptNT), 0, s, a);
    }
  }
  return launch_status();
}

extern "C" aero_status aero_adamw_moments(const void* image, void* table, int32_t dtype, void* avg, void* avg_sq, void* stream) {
  using namespace aero;
  if (!image || !table) return AERO_ERR_NULL;
  const Table* t = table_of(image);
  if (!t) return AERO_ERR_SHAPE;
  if (dtype != AERO_F32 && dtype != AERO_BF16) return AERO_ERR_DTYPE;
  const uint32_t params = t->class_first[class_of(kParamF32, 0, 0)];
  if (t->chunks == params) return AERO_OK;
  if (!avg || !avg_sq) return AERO_ERR_NULL;
  const uintptr_t both = reinterpret_cast<uintptr_t>(avg) | reinterpret_cast<uintptr_t>(avg_sq);
  if (both % storage_bytes(dtype) != 0 || reinterpret_cast<uintptr_t>(table) % 16 != 0) return AERO_ERR_ALIGN;
  hipStream_t s = as_stream(stream);
  for (int k = class_of(kParamF32, 0, 0); k < kClasses; ++k) {
    const uint32_t first = t->class_first[k], chunks = t->class_first[k + 1] - first;
    if (chunks == 0) continue;
    const auto kernel = k % 2 ? (dtype == AERO_F32 ? k_moments<true, kF32> : k_moments<true, kBF16>)
                              : (dtype == AERO_F32 ? k_moments<false, kF32> : k_moments<false, kBF16>);
    for (uint32_t from = 0; from < chunks; from += kMostUnits) {
      const unsigned n = unsigned(chunks - from < kMostUnits ? chunks - from : kMostUnits);
      hipLaunchKernelGGL(kernel, dim3(n), dim3(kOptNT), 0, s, table, t->count, first + from, avg, avg_sq);
    }
  }
  return launch_status();
}
