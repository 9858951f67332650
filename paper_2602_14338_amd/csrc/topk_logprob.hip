// The K largest logits of each row with their log-probs, and the row's log-partition, in one pass over the row.
//
// While the row streams by, each thread notes the largest logit of every group of kGroup of its vectors in LDS (the maximum of a
// vector is formed for the running offset anyway): 152K logits of 16 bits leave 4.7K numbers.  A threshold that at least K
// logits reach follows from the threads' own maxima: each wave removes its lanes' largest ceil(K / waves) times over, and the least of what
// the waves removed last is it.  Groups that reach it, about twice K, are read again, all at once and out of the caches, and
// what reaches it among their logits are the candidates.  A candidate's rank is the count of larger ones; pairs of value and id are
// distinct, so the order is total and ties go to the lower id.
// (Comparing every vector with a threshold from the row's first vectors instead: 900 candidates, a branch in nearly every step of a
// wave, 3.4 times the time of the whole call at 4096 x 151936 bf16.)
// Rows with more candidates than fit (thousands of equal logits at the threshold) are selected digit by digit over their keys, nine more passes.
#include <algorithm>

#include "row_scan.h"

namespace aero {

constexpr int kGroup = 4;            // vectors in flight per thread, and of a group
constexpr int kGroupMax = 5120;      // maxima that are noted; longer rows note one for several groups
constexpr int kCandidates = 1792, kHits = 2048;

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

// A lower bound on the K-th largest logit of the workgroup, from the threads' largest ones (-inf: none); -inf where the
// threads cannot give one.
template <int NT> __device__ float top_threshold(float z, int K, float* lds /*[NT/64]*/) {
  constexpr int kWaves = NT / kWave;
  const int lane = threadIdx.x % kWave;
  const int r = (K + kWaves - 1) / kWaves;
  float least = -INFINITY;
  if (r <= kWave) {
    for (int k = 0; k < r; ++k) {   // uniform
      least = wave_reduce(z, [](float a, float b) { return fmaxf(a, b); });
      const uint64_t with = __builtin_amdgcn_ballot_w64(z == least);
      if (with && lane == __builtin_ctzll(with)) z = -INFINITY;
    }
  }
  if (lane == 0) lds[threadIdx.x / kWave] = least;
  __syncthreads();
  least = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) least = fminf(least, lds[w]);
  return least;
}

struct TopBuffer {
  uint64_t key[kCandidates];
  union {
    float group[kGroupMax];
    uint32_t hist[256];
  };
  uint16_t hit[kHits];
  int count, hits, digit, left;
};

__device__ __forceinline__ void top_push(TopBuffer& b, uint64_t key) {
  const int at = atomicAdd(&b.count, 1);
  if (at < kCandidates) b.key[at] = key;
}

// Exactly the K largest keys of [first, last) of the row (fewer where fewer are unmasked), digit by digit.
template <int NT, int DT, bool VEC>
__device__ __attribute__((noinline)) void top_by_digits(const RowView<DT, VEC>& row, int first, int last, int K, TopBuffer& b) {
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
    __syncthreads();
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
#pragma unroll 8
    for (int k = 0; k < n; ++k) above += b.key[k] > key;
    if (above < K) put(above, key);
  }
}

// Workgroup (t, part): part of the row's vectors.  With one part the outputs; with several the part's keys in descending order (0:
// fewer) and sum for k_topk_join.
template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_topk(const void* __restrict__ logits, int V, int64_t ld, const uint8_t* __restrict__ row_active,
                                             int K, int32_t* __restrict__ index, float* __restrict__ logprob,
                                             float* __restrict__ lse, uint64_t* __restrict__ part_keys, SoftSum* __restrict__ part_sums) {
  constexpr int E = RowView<DT, VEC>::E, kWaves = NT / kWave;
  __shared__ TopBuffer buf;
  __shared__ float s_least[kWaves];
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
  if (tid == 0) {
    buf.count = 0;
    buf.hits = 0;
  }
  const int steps = (last - first + kGroup * NT - 1) / (kGroup * NT);          // of the workgroup
  const int fold = (steps * NT + kGroupMax - 1) / kGroupMax;                   // steps that share a maximum
  const int jr = part == 0 ? row.ragged() : -1;
  const float zr = jr >= 0 ? row.at(jr) : -INFINITY;
  SoftSum st = soft_identity();
  float best = -INFINITY, noted = -INFINITY;
  int i = first + tid;
  for (int step = 0, kept = 0; step < steps; ++step, i += kGroup * NT) {
    u32x4_t v[kGroup];
    if (i + (kGroup - 1) * NT < last) {
#pragma unroll
      for (int u = 0; u < kGroup; ++u) v[u] = row.load(i + u * NT);
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        float z[E];
        row.unpack(v[u], z);
        const float vm = vec_max<E>(z);
        soft_update<E>(st, z, vm);
        noted = fmaxf(noted, vm);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kGroup; ++u)
        if (i + u * NT < last) {
          float z[E];
          row.unpack(row.load(i + u * NT), z);
          const float vm = vec_max<E>(z);
          soft_update<E>(st, z, vm);
          noted = fmaxf(noted, vm);
        }
    }
    if (++kept == fold || step == steps - 1) {
      buf.group[(step / fold) * NT + tid] = noted;
      best = fmaxf(best, noted);
      noted = -INFINITY;
      kept = 0;
    }
  }
  if (jr >= 0) {
    float z[1] = {zr};
    soft_update<1>(st, z);
    best = fmaxf(best, zr);
  }
  const float least = top_threshold<NT>(best > kMasked ? best : -INFINITY, K, s_least);   // its barrier: buf.count, buf.hits
  auto reaches = [&](float z) { return z >= least && z > kMasked; };
  if (reaches(zr)) top_push(buf, top_key(zr, jr));
  if (reaches(best))
    for (int g = 0; g * fold < steps; ++g)
      if (reaches(buf.group[g * NT + tid])) {
        const int at = atomicAdd(&buf.hits, 1);
        if (at < kHits) buf.hit[at] = uint16_t(g * NT + tid);
      }
  st = soft_block_reduce<NT>(st, s_sum);   // its barrier: the hits are complete
  const int hits = buf.hits, span = kGroup * fold;
  if (hits <= kHits)
    for (int k = tid; k < hits * span; k += NT) {
      const int slot = buf.hit[k / span];
      const int vec = first + slot % NT + ((slot / NT) * span + k % span) * NT;
      if (vec < last) {
        float z[E];
        row.unpack(row.load_again(vec), z);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (reaches(z[e])) top_push(buf, top_key(z[e], row.column(vec) + e));
      }
    }
  __syncthreads();
  if (hits > kHits || buf.count > kCandidates) top_by_digits<NT>(row, first, last, K, buf);   // uniform
  const int n = buf.count;
  if (parts > 1) {
    uint64_t* keys = part_keys + (t * parts + part) * K;
    top_rank<NT>(buf, n, K, [&](int r, uint64_t key) { keys[r] = key; });
    for (int k = n + tid; k < K; k += NT) keys[k] = 0;
    if (tid == 0) part_sums[t * parts + part] = st;
    return;
  }
  const double z0 = soft_lse(st);
  top_rank<NT>(buf, n, K, [&](int r, uint64_t key) {
    index[t * K + r] = key_id(key);
    logprob[t * K + r] = float(double(key_logit(key)) - z0);
  });
  for (int k = n + tid; k < K; k += NT) {
    index[t * K + k] = -1;
    logprob[t * K + k] = -INFINITY;
  }
  if (tid == 0 && lse) lse[t] = float(z0);
}

// The parts' lists of a row into one: an entry's rank is its place in its own list and, found by halving, what each other list has
// in front of it.
constexpr int kMaxParts = 8, kJoinNT = 512;
__global__ __launch_bounds__(kJoinNT) void k_topk_join(const uint8_t* __restrict__ row_active, int K, int parts,
                                                       const uint64_t* __restrict__ part_keys, const SoftSum* __restrict__ part_sums,
                                                       int32_t* __restrict__ index, float* __restrict__ logprob,
                                                       float* __restrict__ lse) {
  __shared__ uint64_t s_key[kMaxParts * AERO_TOPK_MAX];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  if (row_active && row_active[t] == 0) return;   // uniform; its outputs were written by its first part
  SoftSum st = soft_identity();
  for (int p = 0; p < parts; ++p) st = soft_merge(st, part_sums[t * parts + p]);
  for (int k = tid; k < parts * K; k += kJoinNT) s_key[k] = part_keys[t * parts * K + k];
  __syncthreads();
  const double z0 = soft_lse(st);
  int mine = 0;
  for (int k = tid; k < parts * K; k += kJoinNT) {
    const uint64_t key = s_key[k];
    if (key == 0) continue;
    ++mine;
    int rank = k % K;
    for (int p = 0; p < parts && rank < K; ++p) {
      if (p == k / K) continue;
      int lo = 0, hi = K;   // entries [0, lo) are above the key, [hi, K) are not
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (s_key[p * K + mid] > key) lo = mid + 1;
        else hi = mid;
      }
      rank += lo;
    }
    if (rank < K) {
      index[t * K + rank] = key_id(key);
      logprob[t * K + rank] = float(double(key_logit(key)) - z0);
    }
  }
  __shared__ int s_n;
  if (tid == 0) s_n = 0;
  __syncthreads();
  if (mine) atomicAdd(&s_n, mine);
  __syncthreads();
  for (int k = s_n + tid; k < K; k += kJoinNT) {
    index[t * K + k] = -1;
    logprob[t * K + k] = -INFINITY;
  }
  if (tid == 0 && lse) lse[t] = float(z0);
}

// Parts of a row.
static int topk_parts(int64_t T, int nvec, int cus) {
  if (T >= 2 * cus || nvec < 2 * kGroup * 256) return 1;
  return int(std::min<int64_t>({kMaxParts, (2 * cus + T - 1) / T, nvec / (kGroup * 256)}));
}

size_t topk_workspace_bytes(int64_t T, int32_t V, int32_t K) {
  (void)V;
  const int64_t rows = std::min<int64_t>(T, 2 * compute_units());   // more are not split
  return size_t(rows) * kMaxParts * (size_t(K > 0 ? K : 0) * 8 + sizeof(SoftSum)) + 256;
}

template <int DT, bool VEC>
static void topk_launch(const void* logits, int64_t T, int V, int64_t ld, const uint8_t* row_active, int K, int32_t* index, float* logprob,
                        float* lse, void* workspace, hipStream_t s) {
  const int nvec = V / RowView<DT, VEC>::E;
  const int parts = topk_parts(T, nvec, compute_units());
  SoftSum* sums = reinterpret_cast<SoftSum*>(workspace);
  uint64_t* keys = reinterpret_cast<uint64_t*>(sums + (parts > 1 ? T * parts : 0));
  const dim3 grid{unsigned(T), unsigned(parts)};
  const int per = (nvec + parts - 1) / parts;
  if (per <= kGroup * 256)
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
  auto launch = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    const auto f = vec ? topk_launch<DT, true> : topk_launch<DT, false>;
    f(logits, T, V, ld, row_active, K, index, logprob, lse, workspace, s);
  };
  switch (dtype) {
    case AERO_BF16: launch(std::integral_constant<int, kBF16>{}); break;
    case AERO_F16: launch(std::integral_constant<int, kF16>{}); break;
    case AERO_F8E4M3: launch(std::integral_constant<int, kF8>{}); break;
    default: launch(std::integral_constant<int, kF32>{});
  }
  return launch_status();
}
