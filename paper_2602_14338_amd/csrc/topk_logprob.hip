// The K largest logits of each row with their log-probs, and the row's log-partition, in one pass over the row.
//
// The first vectors that a workgroup's threads hold give a threshold that at least K of the row's logits reach: each wave removes its
// lanes' largest values ceil(K / waves) times over, and the least of what the waves removed last is it.  The rest
// of the row is only compared with it (the maximum of a vector is formed for the running offset anyway), and what reaches it goes
// into a buffer in LDS: 16 logits of a thread of 151936 in bf16 leave a few hundred.  The rank of a candidate is the count of
// larger ones; pairs of value and id are distinct, so the order is total and ties go to the lower id.
// Rows whose buffer overflows (the large values lie where the threshold did not look) are selected digit by digit over
// their keys, eight more passes, which are found in the caches.
#include "row_scan.h"

namespace aero {

constexpr int kCandidates = 2048;   // capacity of the buffer

// (value, id) as a number that grows with the value and falls with the id; 0: masked or NaN.
__device__ __forceinline__ uint64_t top_key(float z, int j) {
  if (!(z > kMasked)) return 0;
  const uint32_t u = __float_as_uint(z + 0.f);   // -0 and 0 are the same logit
  const uint32_t ord = u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
  return (uint64_t(ord) << 32) | uint32_t(~j);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t ord = uint32_t(key >> 32);
  return __uint_as_float(ord & 0x80000000u ? ord ^ 0x80000000u : ~ord);
}
__device__ __forceinline__ int key_id(uint64_t key) { return int(~uint32_t(key)); }

// A lower bound on the K-th largest key of the workgroup, from one value and id per thread (z = -inf: none).
template <int NT> __device__ uint64_t top_threshold(float z, int j, int K, uint64_t* lds /*[NT/64]*/) {
  constexpr int kWaves = NT / kWave;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int r = (K + kWaves - 1) / kWaves;
  uint64_t least = 0;
  if (r <= kWave) {
    float v = -INFINITY;
    int jmax = 0;
    for (int k = 0; k < r; ++k) {   // uniform
      v = wave_reduce(z, [](float a, float b) { return fmaxf(a, b); });
      const uint64_t with = __builtin_amdgcn_ballot_w64(z == v);
      const int who = with ? __builtin_ctzll(with) : 0;
      jmax = max(jmax, __builtin_amdgcn_readlane(j, who));
      if (lane == who) z = -INFINITY;
    }
    least = top_key(v, jmax);
  }
  if (lane == 0) lds[wave] = least;
  __syncthreads();
  least = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) least = lds[w] < least ? lds[w] : least;
  return least;
}

struct TopBuffer {
  uint64_t key[kCandidates];
  uint32_t hist[256];
  int count, digit, left;
};

__device__ __forceinline__ void top_push(TopBuffer& b, uint64_t key) {
  const int at = atomicAdd(&b.count, 1);
  if (at < kCandidates) b.key[at] = key;
}

// Exactly the K largest keys of [first, last) of the row (fewer where fewer are unmasked), digit by digit.
template <int NT, int DT, bool VEC>
__device__ void top_by_digits(const RowView<DT, VEC>& row, int first, int last, int K, TopBuffer& b) {
  constexpr int E = RowView<DT, VEC>::E;
  const int tid = threadIdx.x;
  const int jr = first == 0 ? row.ragged() : -1;
  auto each = [&](auto f) {
    for (int i = first + tid; i < last; i += NT) {
      float z[E];
      row.unpack(row.load(i), z);
#pragma unroll
      for (int e = 0; e < E; ++e) f(top_key(z[e], row.column(i) + e));
    }
    if (jr >= 0) f(top_key(row.at(jr), jr));
  };
  uint64_t prefix = 0;   // the digits of the K-th key that are known
  int left = K;          // how many keys with this prefix are among the K largest
  for (int shift = 56; shift >= 0; shift -= 8) {
    for (int k = tid; k < 256; k += NT) b.hist[k] = 0;
    __syncthreads();
    each([&](uint64_t key) {
      if (key != 0 && (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8)))) atomicAdd(&b.hist[(key >> shift) & 255], 1u);
    });
    __syncthreads();
    if (tid == 0) {
      int n = left, d = 255;
      while (d > 0 && int(b.hist[d]) < n) n -= int(b.hist[d--]);
      b.digit = d;
      b.left = n;
    }
    __syncthreads();
    prefix |= uint64_t(b.digit) << shift;
    left = b.left;
  }
  if (tid == 0) b.count = 0;
  __syncthreads();
  each([&](uint64_t key) {
    if (key != 0 && key >= prefix) top_push(b, key);
  });
  __syncthreads();
}

// Ranks of the buffer's keys; put(rank, key) for the K first.
template <int NT, class Put> __device__ __forceinline__ void top_rank(const TopBuffer& b, int n, int K, Put put) {
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint64_t key = b.key[i];
    int above = 0;
#pragma unroll 4
    for (int k = 0; k < n; ++k) above += b.key[k] > key;
    if (above < K) put(above, key);
  }
}

// Workgroup (t, part): part of the row's vectors.  With one part the outputs; with several the part's keys (0: fewer) and
// sum for k_topk_join.
template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_topk(const void* __restrict__ logits, int V, int64_t ld, const uint8_t* __restrict__ row_active,
                                             int K, int32_t* __restrict__ index, float* __restrict__ logprob,
                                             float* __restrict__ lse, uint64_t* __restrict__ part_keys, SoftSum* __restrict__ part_sums) {
  constexpr int E = RowView<DT, VEC>::E, kAhead = VEC ? 4 : 8, kWaves = NT / kWave;
  __shared__ TopBuffer buf;
  __shared__ uint64_t s_key[kWaves];
  __shared__ SoftSum s_sum[kWaves];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, parts = gridDim.y, part = blockIdx.y;
  if (row_active && row_active[t] == 0) {
    if (part == 0) {
      for (int k = tid; k < K; k += NT) {
        index[t * K + k] = -1;
        logprob[t * K + k] = 0.f;
      }
      if (tid == 0 && lse) lse[t] = 0.f;
    }
    return;
  }
  const RowView<DT, VEC> row(logits, t, ld, V);
  const int per = (row.nvec + parts - 1) / parts;
  const int first = min(part * per, row.nvec), last = min(first + per, row.nvec);
  if (tid == 0) buf.count = 0;

  // A wave walks a run of its own, so that the vectors in front, which give the threshold, come from all over the part.
  const int run = ((last - first + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int from = first + (tid / kWave) * run, to = min(from + run, last);
  const int i0 = from + tid % kWave;
  const int jr = part == 0 ? row.ragged() : -1;
  const float zr = jr >= 0 ? row.at(jr) : -INFINITY;
  SoftSum st = soft_identity();
  u32x4_t v[kAhead];
  float best = -INFINITY;
  int bj = 0;
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (i0 + u * kWave < to) v[u] = row.load(i0 + u * kWave);
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    if (i0 + u * kWave < to) {
      float z[E];
      row.unpack(v[u], z);
      soft_update<E>(st, z);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (z[e] > best) {
          best = z[e];
          bj = row.column(i0 + u * kWave) + e;
        }
    }
  }
  if (zr > best) {
    best = zr;
    bj = jr;
  }
  const uint64_t least = top_threshold<NT>(best > kMasked ? best : -INFINITY, bj, K, s_key);
  const float lv = least ? key_logit(least) : kMasked;
  const int lj = least ? key_id(least) : -1;
  auto sift = [&](const float (&z)[E], float vm, int j) {
    if (__builtin_amdgcn_ballot_w64(vm >= lv) == 0) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (z[e] > lv || (z[e] == lv && j + e <= lj)) top_push(buf, top_key(z[e], j + e));
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    if (i0 + u * kWave < to) {
      float z[E];
      row.unpack(v[u], z);
      sift(z, vec_max<E>(z), row.column(i0 + u * kWave));
    }
  }
  if (zr > lv || (zr == lv && jr <= lj && jr >= 0)) top_push(buf, top_key(zr, jr));
  if (jr >= 0) {
    float z[1] = {zr};
    soft_update<1>(st, z);
  }
  int i = i0 + kAhead * kWave;
  for (; i + (kAhead - 1) * kWave < to; i += kAhead * kWave) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = row.load(i + u * kWave);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float z[E];
      row.unpack(v[u], z);
      const float vm = vec_max<E>(z);
      soft_update<E>(st, z, vm);
      sift(z, vm, row.column(i + u * kWave));
    }
  }
  for (; i < to; i += kWave) {
    float z[E];
    row.unpack(row.load(i), z);
    const float vm = vec_max<E>(z);
    soft_update<E>(st, z, vm);
    sift(z, vm, row.column(i));
  }
  st = soft_block_reduce<NT>(st, s_sum);   // its barrier: the buffer is complete
  if constexpr (kWaves == 1) __syncthreads();
  if (buf.count > kCandidates) {   // uniform
    __syncthreads();
    top_by_digits<NT>(row, first, last, K, buf);
  }
  const int n = buf.count;
  if (parts > 1) {
    uint64_t* keys = part_keys + (t * parts + part) * K;
    top_rank<NT>(buf, n, K, [&](int r, uint64_t key) { keys[r] = key; });
    for (int k = n + tid; k < K; k += NT) keys[k] = 0;
    if (tid == 0) part_sums[t * parts + part] = st;
    return;
  }
  top_rank<NT>(buf, n, K, [&](int r, uint64_t key) {
    index[t * K + r] = key_id(key);
    logprob[t * K + r] = soft_logprob(st, key_logit(key)).lp;
  });
  for (int k = n + tid; k < K; k += NT) {
    index[t * K + k] = -1;
    logprob[t * K + k] = -INFINITY;
  }
  if (tid == 0 && lse) lse[t] = soft_logprob(st, 0.f).lse;
}

// The parts' lists of a row into one.
constexpr int kJoinNT = 256;
__global__ __launch_bounds__(kJoinNT) void k_topk_join(const uint8_t* __restrict__ row_active, int K, int parts,
                                                       const uint64_t* __restrict__ part_keys, const SoftSum* __restrict__ part_sums,
                                                       int32_t* __restrict__ index, float* __restrict__ logprob,
                                                       float* __restrict__ lse) {
  __shared__ TopBuffer buf;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  if (row_active && row_active[t] == 0) return;   // uniform; its outputs were written by its first part
  SoftSum st = soft_identity();
  for (int p = 0; p < parts; ++p) st = soft_merge(st, part_sums[t * parts + p]);
  if (tid == 0) buf.count = 0;
  __syncthreads();
  for (int k = tid; k < parts * K; k += kJoinNT) {
    const uint64_t key = part_keys[t * parts * K + k];
    if (key != 0) top_push(buf, key);
  }
  __syncthreads();
  const int n = buf.count;
  top_rank<kJoinNT>(buf, n, K, [&](int r, uint64_t key) {
    index[t * K + r] = key_id(key);
    logprob[t * K + r] = soft_logprob(st, key_logit(key)).lp;
  });
  for (int k = n + tid; k < K; k += kJoinNT) {
    index[t * K + k] = -1;
    logprob[t * K + k] = -INFINITY;
  }
  if (tid == 0 && lse) lse[t] = soft_logprob(st, 0.f).lse;
}

// Parts of a row: one (the simple form).
static int topk_parts(int64_t T, int nvec, int K) {
  (void)T;
  (void)nvec;
  (void)K;
  return 1;
}
constexpr int kMaxParts = 8;
static_assert(kMaxParts * AERO_TOPK_MAX <= kCandidates, "the parts' lists fit the buffer");

size_t topk_workspace_bytes(int64_t T, int32_t V, int32_t K) {
  (void)V;
  const int64_t rows = T < 512 ? T : 512;
  return size_t(rows) * kMaxParts * (size_t(K > 0 ? K : 0) * 8 + sizeof(SoftSum)) + 256;
}

template <int DT, bool VEC>
static void topk_launch(const void* logits, int64_t T, int V, int64_t ld, const uint8_t* row_active, int K, int32_t* index, float* logprob,
                        float* lse, void* workspace, hipStream_t s) {
  const int nvec = V / RowView<DT, VEC>::E;
  const int parts = topk_parts(T, nvec, K);
  SoftSum* sums = reinterpret_cast<SoftSum*>(workspace);
  uint64_t* keys = reinterpret_cast<uint64_t*>(sums + (parts > 1 ? T * parts : 0));
  const dim3 grid{unsigned(T), unsigned(parts)};
  const int per = (nvec + parts - 1) / parts;
  if (per <= 4 * 256)
    hipLaunchKernelGGL((k_topk<256, DT, VEC>), grid, dim3(256), 0, s, logits, V, ld, row_active, K, index, logprob, lse, keys, sums);
  else
    hipLaunchKernelGGL((k_topk<512, DT, VEC>), grid, dim3(512), 0, s, logits, V, ld, row_active, K, index, logprob, lse, keys, sums);
  if (parts > 1)
    hipLaunchKernelGGL(k_topk_join, dim3(unsigned(T)), dim3(kJoinNT), 0, s, row_active, K, parts, keys, sums, index, logprob, lse);
}

}  // namespace aero

extern "C" aero_status aero_topk_logprob(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld, const uint8_t* row_active,
                                         int32_t K, int32_t* index, float* logprob, float* lse, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (T < 0 || V < 1 || V > (1 << 24) || ld < V || K < 1 || !grid_fits(T, 1024)) return AERO_ERR_SHAPE;
  if (K > AERO_TOPK_MAX) return AERO_ERR_LIMIT;
  if (!storage_dtype_ok(dtype)) return AERO_ERR_DTYPE;
  if (T == 0) return AERO_OK;
  if (!logits || !index || !logprob) return AERO_ERR_NULL;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < topk_workspace_bytes(T, V, K))
    return AERO_ERR_WORKSPACE;
  const bool vec = rows_alike(logits, nullptr, storage_bytes(dtype));
  const hipStream_t s = as_stream(stream);
#define AERO_TOPK(DT)                                                                                       \
  vec ? topk_launch<DT, true>(logits, T, V, ld, row_active, K, index, logprob, lse, workspace, s)          \
      : topk_launch<DT, false>(logits, T, V, ld, row_active, K, index, logprob, lse, workspace, s)
  switch (dtype) {
    case AERO_BF16: AERO_TOPK(kBF16); break;
    case AERO_F16: AERO_TOPK(kF16); break;
    case AERO_F8E4M3: AERO_TOPK(kF8); break;
    default: AERO_TOPK(kF32);
  }
#undef AERO_TOPK
  return launch_status();
}
