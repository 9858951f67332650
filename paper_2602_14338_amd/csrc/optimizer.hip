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
constexpr int kOptNT = 256, kPer = 8, kChunk = kOptNT * kPer, kBlock = AERO_MOMENT_BLOCK;
static_assert(kBlock == 32 * kPer, "half a wave holds a block of moments");

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

constexpr uint64_t kMagic = 0x41455254'61626c65ull;
struct Table {
  uint64_t magic;
  uint64_t bytes;
  int32_t count;
  uint32_t chunks;
  uint32_t ticket;        // of the step's workgroups (device copy)
  uint32_t pad;
  uint32_t class_first[kClasses + 1];   // chunks of class k: class_first[k] .. class_first[k + 1]
  uint32_t pad2;
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
// Eight stored elements at any alignment as 32-bit floats.
template <int DT> __device__ __forceinline__ void load8(const void* base, uint64_t i, float (&x)[kPer]) {
  const char* p = static_cast<const char*>(base) + i * Storage<DT>::kBytes;
  if constexpr (DT == kF32) {
    const f32x4_any_t a = reinterpret_cast<const f32x4_any_t*>(p)[0], b = reinterpret_cast<const f32x4_any_t*>(p)[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = a[k], x[4 + k] = b[k];
  } else {
    const u32x4_any_t a = *reinterpret_cast<const u32x4_any_t*>(p);
    unpack_vec<DT>(u32x4_t{a.x, a.y, a.z, a.w}, x);
  }
}
template <int DT> __device__ __forceinline__ void store8(void* base, uint64_t i, const float (&x)[kPer]) {
  char* p = static_cast<char*>(base) + i * Storage<DT>::kBytes;
  if constexpr (DT == kF32) {
    f32x4_any_t a, b;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = x[k], b[k] = x[4 + k];
    reinterpret_cast<f32x4_any_t*>(p)[0] = a;
    reinterpret_cast<f32x4_any_t*>(p)[1] = b;
  } else {
    const u32x4_t v = pack_vec<DT>(x);
    *reinterpret_cast<u32x4_any_t*>(p) = u32x4_any_t{v.x, v.y, v.z, v.w};
  }
}
// The same up to a tensor's end: `have` elements of the eight (others read as 0).
template <int DT> __device__ __forceinline__ void load_upto(const void* base, uint64_t i, int have, float (&x)[kPer]) {
  if (have >= kPer) return load8<DT>(base, i, x);
#pragma unroll
  for (int k = 0; k < kPer; ++k) x[k] = k < have ? load_elt<DT>(base, int64_t(i) + k) : 0.f;
}
template <int DT> __device__ __forceinline__ void store_upto(void* base, uint64_t i, int have, const float (&x)[kPer]) {
  if (have >= kPer) return store8<DT>(base, i, x);
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (k < have) store_elt<DT>(base, int64_t(i) + k, x[k]);
}
__device__ __forceinline__ void load_codes(const char* base, uint64_t i, int have, uint32_t (&w)[2]) {
  if (have >= kPer) {
    const u32x2_any_t v = *reinterpret_cast<const u32x2_any_t*>(base + i);
    w[0] = v.x;
    w[1] = v.y;
    return;
  }
  w[0] = w[1] = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (k < have) w[k / 4] |= uint32_t(uint8_t(base[i + k])) << (8 * (k % 4));
}
__device__ __forceinline__ void store_codes(char* base, uint64_t i, int have, const uint32_t (&w)[2]) {
  if (have >= kPer) {
    *reinterpret_cast<u32x2_any_t*>(base + i) = u32x2_any_t{w[0], w[1]};
    return;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (k < have) base[i + k] = char(w[k / 4] >> (8 * (k % 4)));
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
template <bool FIRST> __device__ __forceinline__ void decode8(const uint32_t (&w)[2], float scale, float (&x)[kPer]) {
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if constexpr (FIRST) x[k] = first_value(float(int8_t(w[k / 4] >> (8 * (k % 4)))), scale);
    else x[k] = second_value(float(w[k / 4] >> (8 * (k % 4)) & 0xff), scale);
  }
}
// The largest of a block's 256 moments by its bits (as whole numbers infinities and NaN come out largest): half a wave.
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
  auto most = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  x = most(x, uint32_t(dpp_move_i<0xB1>(int(x))));
  x = most(x, uint32_t(dpp_move_i<0x4E>(int(x))));
  x = most(x, uint32_t(dpp_move_i<0x141>(int(x))));
  x = most(x, uint32_t(dpp_move_i<0x140>(int(x))));
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return most(r[0], r[1]);
}
__device__ __forceinline__ float block_scale(const float (&x)[kPer], float inv_top) {
#pragma clang fp contract(off)
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const uint32_t b = __float_as_uint(x[k]) & 0x7fffffffu;
    most = b > most ? b : most;
  }
  most = block_max(most);
  if (most >= 0x7f800000u) return __builtin_nanf("");
  const float s = __uint_as_float(most) * inv_top;
  return s >= 1.17549435e-38f ? s : 0.f;
}
__device__ __forceinline__ int first_code(float x, float inv, float u) {
#pragma clang fp contract(off)
  const float y = fminf(fabsf(x) * inv, kTop1);
  float c = floorf(__builtin_amdgcn_sqrtf(y));
  if (c * c > y) c -= 1.f;
  else if ((c + 1.f) * (c + 1.f) <= y) c += 1.f;
  if (u * (2.f * c + 1.f) < y - c * c) c += 1.f;
  return int(x < 0.f ? -c : c);
}
__device__ __forceinline__ uint32_t second_code(float x, float inv, float u) {
#pragma clang fp contract(off)
  const float y = fminf(x * inv, kTop2);
  float c = floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(y)));
  if (fourth(c) > y) c -= 1.f;
  else if (fourth(c + 1.f) <= y) c += 1.f;
  const float at = fourth(c);
  if (u * (fourth(c + 1.f) - at) < y - at) c += 1.f;
  return uint32_t(y > 0.f ? fminf(fmaxf(c, 1.f), 255.f) : 0.f);
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
  uint32_t first, chunks;   // of this launch's class
  int32_t last;             // counts the step
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

template <int KIND, int GRAD, bool SMALL>
__global__ __launch_bounds__(kOptNT) void k_adamw(StepArgs a) {
  const float factor = a.factor ? a.factor[0] : 1.f;
  const int step = a.step[0];
  if (!(fabsf(factor) < INFINITY)) return;   // uniform over the launch
  const uint32_t t = uint32_t(step) + 1;
  const double rate = a.lr * (a.lr_factor ? double(a.lr_factor[0]) : 1.0);
  const float by_first = float(rate / (1.0 - power(a.dbeta1, t)));
  const float by_second = float(1.0 / sqrt(1.0 - power(a.dbeta2, t)));
  const uint32_t of_step = mix(a.seed_lo ^ mix(a.seed_hi ^ mix(uint32_t(step))));
  const Tensor* tensors = tensors_of(a.table);
  const uint32_t* map = map_of(a.table, a.count);
  constexpr bool kMaster = KIND == kMasterBF16 || KIND == kMasterF16;
  constexpr int kStored = KIND == kParamF32 ? kF32 : KIND == kMasterF16 ? kF16 : kBF16;
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Tensor& e = tensors[__builtin_amdgcn_readfirstlane(map[a.first + c])];
    const uint64_t i = uint64_t(a.first + c - e.first_chunk) * kChunk + threadIdx.x * kPer;
    const int64_t behind = e.n - int64_t(i);
    const int have = behind >= kPer ? kPer : behind > 0 ? int(behind) : 0;
    float p[kPer], g[kPer], m[kPer], v[kPer];
    load_upto<GRAD>(e.grad, i, have, g);
    if constexpr (kMaster) load_upto<kF32>(e.master, i, have, p);
    else load_upto<kStored>(e.param, i, have, p);
    if constexpr (SMALL) {
      uint32_t wm[2], wv[2];
      load_codes(e.avg, i, have, wm);
      load_codes(e.sq, i, have, wv);
      const uint64_t block = i / kBlock;
      const bool in = have > 0;
      decode8<true>(wm, in ? e.avg_scale[block] : 0.f, m);
      decode8<false>(wv, in ? e.sq_scale[block] : 0.f, v);
    } else {
      load_upto<kF32>(e.avg, i, have, m);
      load_upto<kF32>(e.sq, i, have, v);
    }
    const float keep = float(1.0 - rate * a.weight_decay * double(e.decay));
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
#pragma clang fp contract(off)
      const float x = g[k] * factor;
      m[k] = m[k] * a.beta1 + x * a.beta1c;
      v[k] = v[k] * a.beta2 + (x * x) * a.beta2c;
      const float away = sqrtf(v[k]) * by_second + a.eps;
      p[k] = p[k] * keep - m[k] / away * by_first;
    }
    const bool random_param = KIND == kParamBF16 && a.stochastic;
    uint32_t bits[kPer];
    if ((SMALL || KIND == kParamBF16) && a.stochastic) {
      const uint32_t of_tensor = mix(of_step + uint32_t(e.ordinal));
#pragma unroll
      for (int k = 0; k < kPer; ++k) bits[k] = mix(of_tensor + uint32_t(i) + uint32_t(k));
    }
    if constexpr (SMALL) {
      const float sm = block_scale(m, kInvTop1), sv = block_scale(v, kInvTop2);
      const float im = sm > 0.f ? 1.f / sm : 0.f, iv = sv > 0.f ? 1.f / sv : 0.f;
      uint32_t wm[2] = {0, 0}, wv[2] = {0, 0};
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const float um = a.stochastic ? uniform16(bits[k] & 0xffff) : 0.5f, uv = a.stochastic ? uniform16(bits[k] >> 16) : 0.5f;
        wm[k / 4] |= (uint32_t(first_code(m[k], im, um)) & 0xff) << (8 * (k % 4));
        wv[k / 4] |= second_code(v[k], iv, uv) << (8 * (k % 4));
      }
      store_codes(e.avg, i, have, wm);
      store_codes(e.sq, i, have, wv);
      if (have > 0 && threadIdx.x % 32 == 0) {
        e.avg_scale[i / kBlock] = sm;
        e.sq_scale[i / kBlock] = sv;
      }
    } else {
      store_upto<kF32>(e.avg, i, have, m);
      store_upto<kF32>(e.sq, i, have, v);
    }
    if constexpr (kMaster) store_upto<kF32>(e.master, i, have, p);
    if (random_param) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const uint32_t raw = __float_as_uint(p[k]);
        if ((raw & 0x7f800000u) != 0x7f800000u) p[k] = __uint_as_float((raw + (bits[k] * 0x9E3779B1u >> 16)) & 0xffff0000u);
      }
    }
    store_upto<kStored>(e.param, i, have, p);
  }
  // the last workgroup to end counts the step: by then every wave of every workgroup has read it
  if (!a.last) return;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t* ticket = &static_cast<Table*>(a.table)->ticket;
    if (atomicAdd(ticket, 1u) == gridDim.x - 1) {
      *ticket = 0;
      a.step[0] = step + 1;
    }
  }
}

// A table without parameters still counts its steps.
__global__ void k_count_step(int32_t* step, const float* factor) {
  if (!factor || fabsf(factor[0]) < INFINITY) step[0] += 1;
}

using StepKernel = void (*)(StepArgs);
template <int KIND, int GRAD> static StepKernel step_kernel(bool small) { return small ? k_adamw<KIND, GRAD, true> : k_adamw<KIND, GRAD, false>; }
template <int KIND> static StepKernel step_kernel(int grad, bool small) {
  return grad == 0 ? step_kernel<KIND, kF32>(small) : grad == 1 ? step_kernel<KIND, kBF16>(small) : step_kernel<KIND, kF16>(small);
}
static StepKernel step_kernel(int cls) {
  const int kind = cls / 2 / kGrads, grad = cls / 2 % kGrads;
  const bool small = cls % 2;
  switch (kind) {
    case kParamF32: return step_kernel<kParamF32>(grad, small);
    case kParamBF16: return step_kernel<kParamBF16>(grad, small);
    case kMasterBF16: return step_kernel<kMasterBF16>(grad, small);
    default: return step_kernel<kMasterF16>(grad, small);
  }
}

// ---------------------------------------------------------------------------------- moments as numbers
template <bool SMALL, int DT>
__global__ __launch_bounds__(kOptNT) void k_moments(void* table, int32_t count, uint32_t first, uint32_t chunks, void* avg, void* sq) {
  const Tensor* tensors = tensors_of(table);
  const uint32_t* map = map_of(table, count);
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Tensor& e = tensors[__builtin_amdgcn_readfirstlane(map[first + c])];
    const uint64_t i = uint64_t(first + c - e.first_chunk) * kChunk + threadIdx.x * kPer;
    const int64_t behind = e.n - int64_t(i);
    const int have = behind >= kPer ? kPer : behind > 0 ? int(behind) : 0;
    if (have == 0) continue;
    float m[kPer], v[kPer];
    if constexpr (SMALL) {
      uint32_t w[2];
      load_codes(e.avg, i, have, w);
      decode8<true>(w, e.avg_scale[i / kBlock], m);
      load_codes(e.sq, i, have, w);
      decode8<false>(w, e.sq_scale[i / kBlock], v);
    } else {
      load_upto<kF32>(e.avg, i, have, m);
      load_upto<kF32>(e.sq, i, have, v);
    }
    store_upto<DT>(avg, uint64_t(e.out) + i, have, m);
    store_upto<DT>(sq, uint64_t(e.out) + i, have, v);
  }
}

// ---------------------------------------------------------------------------------- norm
constexpr int kNormMax = 2048;   // workgroups
template <int DT> __device__ __forceinline__ void add_squares(const Tensor& e, uint64_t i, int have, double& sum) {
  float g[kPer];
  load_upto<DT>(e.grad, i, have, g);
#pragma unroll
  for (int k = 0; k < kPer; ++k) sum = fma(double(g[k]), double(g[k]), sum);
}
__global__ __launch_bounds__(kOptNT) void k_norm_parts(const void* table, int32_t count, uint32_t chunks, double* __restrict__ part) {
  const Tensor* tensors = tensors_of(table);
  const uint32_t* map = map_of(table, count);
  double sum = 0.0;
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Tensor& e = tensors[__builtin_amdgcn_readfirstlane(map[c])];
    const uint64_t i = uint64_t(c - e.first_chunk) * kChunk + threadIdx.x * kPer;
    const int64_t behind = e.n - int64_t(i);
    const int have = behind >= kPer ? kPer : behind > 0 ? int(behind) : 0;
    const int grad = e.kind / 2 % kGrads;
    if (grad == 0) add_squares<kF32>(e, i, have, sum);
    else if (grad == 1) add_squares<kBF16>(e, i, have, sum);
    else add_squares<kF16>(e, i, have, sum);
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
  if (chunks >= (uint64_t(1) << 31)) return AERO_ERR_SHAPE;
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
  int last = -1;
  for (int k = class_of(kParamF32, 0, 0); k < kClasses; ++k)
    if (t->class_first[k + 1] > t->class_first[k]) last = k;
  if (last < 0) {
    hipLaunchKernelGGL(k_count_step, dim3(1), dim3(1), 0, s, step, factor);
    return launch_status();
  }
  for (int k = class_of(kParamF32, 0, 0); k <= last; ++k) {
    a.first = t->class_first[k];
    a.chunks = t->class_first[k + 1] - a.first;
    if (a.chunks == 0) continue;
    a.last = k == last;
    hipLaunchKernelGGL(step_kernel(k), dim3(opt_grid(a.chunks, 8)), dim3(kOptNT), 0, s, a);
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
    hipLaunchKernelGGL(kernel, dim3(opt_grid(chunks, 8)), dim3(kOptNT), 0, s, table, t->count, first, chunks, avg, avg_sq);
  }
  return launch_status();
}
