// The K largest logits of each row with their log-probs, and the row's log-partition, in one pass over the row.
//
// A short row is held in registers.  While a long one streams by, each thread notes the largest logit of every kGroup of its vectors in
// LDS, 16 bits of it (the maximum of a vector is formed for the running offset anyway): 152K logits of 16 bits leave 9.5K numbers.  A threshold that at least
// K logits reach follows from the threads' own maxima, joined into about 2 K of them: the K-th largest of these, found bit by bit by one wave.
// Groups that reach it, little more than K, are read again, all at once and out of the caches, and what reaches it among their logits are the
// candidates.  A candidate's rank is the count of larger ones, of which only those in its own interval of values are gone through where there
// are many (all pairs instead: 4000 rows of 2399, K = 120 and 256, 35 and 101 us for 20 and 41); pairs of value and id are distinct, so the order is
// total and ties go to the lower id.
// (Comparing every vector with a threshold from the row's first vectors instead: 900 candidates, a branch in nearly every step of a
// wave, 3.4 times the time of the whole call at 4096 x 151936 bf16.)
// Rows with more candidates than fit (thousands of equal logits at the threshold) are selected digit by digit over their keys, nine more passes.
// Bound by the row's bytes where there are many: 4096 x 151936 bf16, K = 64, 201 us (6.2 TB/s); by the chain of load, threshold, candidates and
// ranks (10000 cycles of a short row) and a second launch where there are few: 64 such rows, in four parts each, 16.3 us.
#include <algorithm>
#include <type_traits>

#include "row_scan.h"

namespace aero {

constexpr int kGroup = 2, kAhead = 2;   // vectors of a group, groups of a batch
// Maxima that are noted; longer rows note one for several groups.
constexpr int group_max(int threads) { return threads == 256 ? 2048 : 10240; }
constexpr int kCandidates = 1536, kHits = 1024;
constexpr int kBins = 256;
constexpr int kPairs = 16;   // comparisons of a thread up to which all pairs of candidates are as fast as intervals

// The order of floats as that of whole numbers; -0 and 0 are the same.
__device__ __forceinline__ uint32_t float_order(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_float(uint32_t ord) { return __uint_as_float(ord & 0x80000000u ? ord ^ 0x80000000u : ~ord); }

// (value, id) as a number that grows with the value and falls with the id; 0: masked or NaN.
__device__ __forceinline__ uint64_t top_key(float z, int j) {
  if (!(z > kMasked)) return 0;
  return (uint64_t(float_order(z)) << 32) | uint32_t(~j);
}
__device__ __forceinline__ float key_logit(uint64_t key) { return order_float(uint32_t(key >> 32)); }
__device__ __forceinline__ int key_id(uint64_t key) { return int(~uint32_t(key)); }

// A lower bound on the K-th largest of the NT numbers in `best` (-inf: none), -inf where there are no K of them; by one wave.  They are joined
// into N x 64 maxima, K <= 32 N, of which at least as many reach it: for K = 64 joining 512 into 128 makes 89 of 68 candidates, and only
// one wave counts (16 waves that each count their own lanes share the CU's one scalar unit: 6 times as long).  Bit by bit, from the
// counts of lanes that reach a number; 18 bits tell all 16- and 8-bit logits apart and leave a bound for the others.
template <int NT, int N> __device__ __forceinline__ float top_threshold(const float* best, int K) {
  constexpr int kJoined = NT / (kWave * N);
  uint32_t ord[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float most = best[n * kWave + threadIdx.x];
#pragma unroll
    for (int j = 1; j < kJoined; ++j) most = fmaxf(most, best[(j * N + n) * kWave + threadIdx.x]);
    ord[n] = float_order(most);
  }
  uint32_t reached = 0;
#pragma unroll
  for (int shift = 31; shift >= 14; --shift) {
    int lanes = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) lanes += __popcll(__builtin_amdgcn_ballot_w64(ord[n] >= (reached | 1u << shift)));
    if (lanes >= K) reached |= 1u << shift;
  }
  const float least = order_float(reached);   // without a logit: at or below -inf's bits
  return least > kMasked ? least : -INFINITY;
}
template <int NT> __device__ __forceinline__ float top_threshold_of(const float* best, int K) {
  constexpr int kMost = NT / kWave;
  if (K <= 32) return top_threshold<NT, 1>(best, K);   // uniform
  if (K <= 64) return top_threshold<NT, 2>(best, K);
  if (K <= 128) return top_threshold<NT, 4>(best, K);
  return top_threshold<NT, kMost < 8 ? kMost : 8>(best, K);
}

struct TopBuffer {
  uint64_t key[kCandidates];
  alignas(16) uint32_t hist[kBins];
  int count, digit, left;
};
// What is noted while a row streams by.
template <int NT> struct TopGroups {
  uint16_t most[group_max(NT)];   // upper halves of the maxima
  uint16_t hit[kHits];
  int hits;
};
struct NoGroups {};

__device__ __forceinline__ void top_push(TopBuffer& b, uint64_t key) {
  const int at = atomicAdd(&b.count, 1);
  if (at < kCandidates) b.key[at] = key;
}

// Pushes the logits of U vectors (column -1: none) that reach `least`, behind one count of the wave's (a count for each: 150 cycles one
// after the other).  By whole waves.
template <int U, class View> __device__ __forceinline__ void top_push(TopBuffer& b, const View& row, const u32x4_t (&v)[U], const int (&column)[U], float least) {
  constexpr int E = View::E;
  auto each = [&](auto f) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float z[E];
      row.unpack(v[u], z);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (column[u] >= 0 && z[e] >= least && z[e] > kMasked) f(z[e], column[u] + e);
    }
  };
  int n = 0;
  each([&](float, int) { ++n; });
  if (__builtin_amdgcn_ballot_w64(n > 0) == 0) return;
  const int up_to = int(wave_scan(uint32_t(n)));
  int at = 0;
  if (threadIdx.x % kWave == kWave - 1) at = atomicAdd(&b.count, up_to);
  at = __builtin_amdgcn_readlane(at, kWave - 1) + up_to - n;
  each([&](float z, int j) {
    if (at < kCandidates) b.key[at] = top_key(z, j);
    ++at;
  });
}

// Exactly the K largest keys of [first, last) of the row (fewer where fewer are unmasked), digit by digit.  In place: a call, rare as it
// is, gives the kernel a stack, and a launch whose waves need one starts them so slowly that 4096 rows take 240 us for 200.
template <int NT, int DT, bool VEC>
__device__ __forceinline__ void top_by_digits(const RowView<DT, VEC>& row, int first, int last, int K, TopBuffer& b) {
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
    for (int k = tid; k < kBins; k += NT) b.hist[k] = 0;
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

// Ranks of the buffer's keys; put(rank, key) for the K first.  As many threads share a key as there are for each.
template <int NT, class Put> __device__ __forceinline__ void top_rank(const TopBuffer& b, int n, int K, Put put) {
  int share = 1;
  while (share < 16 && 2 * share * n <= NT) share *= 2;   // uniform; threads that share a key are in one row of 16 lanes
  const int sub = threadIdx.x % share;
  for (int i0 = 0; i0 < n; i0 += NT / share) {
    const int i = i0 + threadIdx.x / share;
    const uint64_t key = i < n ? b.key[i] : ~uint64_t(0);
    int above = 0;
#pragma unroll 4
    for (int k = sub; k < n; k += share) above += b.key[k] > key;
    if (share > 1) above += dpp_move_i<0xB1>(above);
    if (share > 2) above += dpp_move_i<0x4E>(above);
    if (share > 4) above += dpp_move_i<0x141>(above);   // the mirrors stand for exchanges at distance 4 and 8
    if (share > 8) above += dpp_move_i<0x140>(above);
    if (sub == 0 && i < n && above < K) put(above, key);
  }
}

// A part of a row that streams by: its sum, and the largest logit of every group noted.
template <int NT, int DT, bool VEC> struct Streamed {
  using View = RowView<DT, VEC>;
  static constexpr int E = View::E;
  const View& row;
  const int first, last;
  TopGroups<NT>& groups;
  const int tid = threadIdx.x;
  const int steps = (last - first + kGroup * NT - 1) / (kGroup * NT);                    // of the workgroup
  const int fold = max((steps * NT + group_max(NT) - 1) / group_max(NT), 1);             // steps that share a maximum

  __device__ __forceinline__ void read(SoftSum& st, float& best) {
    float noted = -INFINITY;
    int i = first + tid;
    int step = 0, kept = 0, slot = tid;
    auto note = [&]() {   // the end of a step
      ++step;
      if (++kept == fold || step == steps) {
        groups.most[slot] = uint16_t(__float_as_uint(noted) >> 16);
        slot += NT;
        best = fmaxf(best, noted);
        noted = -INFINITY;
        kept = 0;
      }
    };
    auto take = [&](const u32x4_t& x) {
      float z[E];
      row.unpack(x, z);
      const float vm = vec_max<E>(z);
      soft_update<E>(st, z, vm);
      noted = fmaxf(noted, vm);
    };
    // batches of kAhead groups, the next one asked for before this one is used
    constexpr int kBatch = kAhead * kGroup;
    u32x4_t ahead[kBatch];
    auto ask = [&](u32x4_t (&v)[kBatch]) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) v[u] = row.load(i + u * NT);
    };
    bool more = i + (kBatch - 1) * NT < last;
    if (more) ask(ahead);
    while (more) {
      u32x4_t v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) v[u] = ahead[u];
      i += kBatch * NT;
      more = i + (kBatch - 1) * NT < last;
      if (more) ask(ahead);
#pragma unroll
      for (int g = 0; g < kAhead; ++g) {   // one test of the offset for a group
        float z[kGroup * E];
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
          float x[E];
          row.unpack(v[g * kGroup + u], x);
#pragma unroll
          for (int e = 0; e < E; ++e) z[u * E + e] = x[e];
        }
        const float vm = vec_max<kGroup * E>(z);
        soft_update<kGroup * E>(st, z, vm);
        noted = fmaxf(noted, vm);
        note();
      }
    }
    while (step < steps) {   // note() counts
      u32x4_t v[kGroup];
#pragma unroll
      for (int u = 0; u < kGroup; ++u)
        if (i + u * NT < last) v[u] = row.load(i + u * NT);
#pragma unroll
      for (int u = 0; u < kGroup; ++u)
        if (i + u * NT < last) take(v[u]);
      note();
      i += kGroup * NT;
    }
  }
  // Pushes what reaches `least`; false where the groups that do are more than are listed.  By all threads.
  __device__ __forceinline__ bool push(TopBuffer& buf, float best, float least) {
    auto reaches = [&](float z) { return z >= least && z > kMasked; };
    // ---- groups that reach the threshold: cutting off lower halves keeps the order ----
    if (reaches(best)) {
      const float bound = __uint_as_float(__float_as_uint(least) & 0xffff0000u);
      const int mine = (steps + fold - 1) / fold;
      for (int g0 = 0; g0 < mine; g0 += 4) {
        uint32_t code[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) code[u] = groups.most[min(g0 + u, mine - 1) * NT + tid];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float most = __uint_as_float(code[u] << 16);
          if (g0 + u < mine && most >= bound && most > kMasked) {
            const int at = atomicAdd(&groups.hits, 1);
            if (at < kHits) groups.hit[at] = uint16_t((g0 + u) * NT + tid);
          }
        }
      }
    }
    __syncthreads();
    // ---- their logits ----
    const int hits = groups.hits, span = kGroup * fold;
    if (hits > kHits) return false;
    for (int k0 = 0; k0 < hits * span; k0 += 4 * NT) {
      u32x4_t v[4];
      int vec[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = min(k0 + u * NT + tid, hits * span - 1), slot = groups.hit[k / span];
        vec[u] = first + slot % NT + ((slot / NT) * span + k % span) * NT;
        if (k0 + u * NT + tid >= hits * span || vec[u] >= last) vec[u] = -1;
        v[u] = row.load_again(max(vec[u], 0));
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float z[E];
        row.unpack(v[u], z);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (vec[u] >= 0 && reaches(z[e])) top_push(buf, top_key(z[e], row.column(vec[u]) + e));
      }
    }
    return true;
  }
};

// A part of at most N vectors per thread, which hold it.
template <int NT, int DT, bool VEC, int N> struct Held {
  using View = RowView<DT, VEC>;
  static constexpr int E = View::E;
  const View& row;
  const int first, last;
  NoGroups& groups;
  u32x4_t v[N];

  template <class F> __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int k = first + int(threadIdx.x) + u * NT;
      if (k < last) f(v[u], k);
    }
  }
  __device__ __forceinline__ void read(SoftSum& st, float& best) {
    each([&](u32x4_t& x, int k) { x = row.load(k); });
    float z[E];
    each([&](const u32x4_t& x, int) {
      row.unpack(x, z);
      best = fmaxf(best, vec_max<E>(z));
    });
    if (best > kMasked) st.o = soft_offset(best);
    each([&](const u32x4_t& x, int) {
      row.unpack(x, z);
      soft_add<E>(st, z);
    });
  }
  __device__ __forceinline__ bool push(TopBuffer& buf, float best, float least) {
    if (__builtin_amdgcn_ballot_w64(best >= least && best > kMasked) == 0) return true;
    int column[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int k = first + int(threadIdx.x) + u * NT;
      column[u] = k < last ? row.column(k) : -1;
    }
    top_push(buf, row, v, column, least);
    return true;
  }
};

// The same for many keys: they are dealt out over kBins intervals of [least, most], largest first, and ranked within theirs.
template <int NT, class Put> __device__ __forceinline__ void top_rank_binned(TopBuffer& b, int n, int K, float least, float most, Put put) {
  constexpr int kEach = (kCandidates + NT - 1) / NT;
  const int tid = threadIdx.x;
  const float scale = float(kBins) / (most - least);
  uint64_t key[kEach];
  int bin[kEach], at[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int i = tid + u * NT;
    if (i < n) {
      key[u] = b.key[i];
      bin[u] = int(fminf(fmaxf((most - key_logit(key[u])) * scale, 0.f), float(kBins - 1)));   // falls with the logit; NaN: 0
      at[u] = atomicAdd(&b.hist[bin[u]], 1u);
    }
  }
  __syncthreads();
  if (tid < kWave) {   // counts into the first places
    static_assert(kBins == 4 * kWave, "four intervals a lane");
    u32x4_t* const mine = reinterpret_cast<u32x4_t*>(b.hist) + tid;
    const u32x4_t x = *mine;
    const uint32_t all = x.x + x.y + x.z + x.w, before = wave_scan(all) - all;
    *mine = u32x4_t{before, before + x.x, before + x.x + x.y, before + x.x + x.y + x.z};
  }
  __syncthreads();
  int first[kEach], end[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u)
    if (tid + u * NT < n) {
      first[u] = int(b.hist[bin[u]]);
      end[u] = bin[u] + 1 < kBins ? int(b.hist[bin[u] + 1]) : n;
      b.key[first[u] + at[u]] = key[u];
    }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kEach; ++u)
    if (tid + u * NT < n) {
      int rank = first[u];
#pragma unroll 4
      for (int k = first[u]; k < end[u]; ++k) rank += b.key[k] > key[u];
      if (rank < K) put(rank, key[u]);
    }
}

// Workgroup (t, part): part of the row's vectors.  With one part the outputs; with several the part's keys in descending order (0:
// fewer) and sum for k_topk_join.
template <int NT, int DT, bool VEC, int HELD>   // vectors that a thread holds, 0: the row streams by
__global__ __launch_bounds__(NT) void k_topk(const void* __restrict__ logits, int V, int64_t ld, const uint8_t* __restrict__ row_active,
                                             int K, int32_t* __restrict__ index, float* __restrict__ logprob,
                                             float* __restrict__ lse, uint64_t* __restrict__ part_keys, SoftSum* __restrict__ part_sums) {
  constexpr int kWaves = NT / kWave;
  using Part = std::conditional_t<HELD != 0, Held<NT, DT, VEC, HELD>, Streamed<NT, DT, VEC>>;
  __shared__ TopBuffer buf;
  __shared__ std::conditional_t<HELD != 0, NoGroups, TopGroups<NT>> groups;
  __shared__ float s_best[NT], s_least, s_most;
  __shared__ double s_lse;
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
  for (int k = tid; k < kBins; k += NT) buf.hist[k] = 0;
  if (tid == 0) {
    buf.count = 0;
    if constexpr (HELD == 0) groups.hits = 0;
  }
  const int jr = part == 0 ? row.ragged() : -1;
  const float zr = jr >= 0 ? row.at(jr) : -INFINITY;
  SoftSum st = soft_identity();
  float best = -INFINITY;
  Part mine{row, first, last, groups};
  mine.read(st, best);
  if (jr >= 0) {
    float z[1] = {zr};
    soft_update<1>(st, z);
    best = fmaxf(best, zr);
  }
  s_best[tid] = best > kMasked ? best : -INFINITY;
  st = soft_block_reduce<NT>(st, s_sum);   // its barrier: s_best
  if (tid < kWave) {
    const float reached = top_threshold_of<NT>(s_best, K);
    if (tid == 0) s_least = reached;
  } else if (tid >= NT - kWave) {   // beside it
    const double z0 = soft_lse(st);
    if (tid == NT - 1) s_lse = z0;
  } else if (tid >= NT - 2 * kWave) {
    float most = s_best[tid % kWave];
#pragma unroll
    for (int k = 1; k < NT / kWave; ++k) most = fmaxf(most, s_best[k * kWave + tid % kWave]);
    most = wave_reduce(most, [](float x, float y) { return fmaxf(x, y); });
    if (tid == NT - 2 * kWave) s_most = most;
  }
  __syncthreads();
  const float least = s_least;
  if (zr >= least && zr > kMasked) top_push(buf, top_key(zr, jr));
  const bool listed = mine.push(buf, best, least);
  __syncthreads();
  const bool digits = !listed || buf.count > kCandidates;   // uniform
  if (digits) top_by_digits<NT>(row, first, last, K, buf);
  const int n = buf.count;
  auto rank = [&](auto put) {
    if (digits || n * n < kPairs * NT) top_rank<NT>(buf, n, K, put);
    else top_rank_binned<NT>(buf, n, K, least, s_most, put);
  };
  if (parts > 1) {
    uint64_t* keys = part_keys + (t * parts + part) * K;
    rank([&](int r, uint64_t key) { keys[r] = key; });
    for (int k = n + tid; k < K; k += NT) keys[k] = 0;
    if (tid == 0) part_sums[t * parts + part] = st;
    return;
  }
  const double z0 = s_lse;
  rank([&](int r, uint64_t key) {
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
  __shared__ double s_lse;
  __shared__ int s_n;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  if (row_active && row_active[t] == 0) return;   // uniform; its outputs were written by its first part
  SoftSum st = soft_identity();
  if (tid >= kJoinNT - kWave && tid % 16 < parts) st = part_sums[t * parts + tid % 16];
  if (tid == 0) s_n = 0;
  for (int k = tid; k < parts * K; k += kJoinNT) s_key[k] = part_keys[t * parts * K + k];
  if (tid >= kJoinNT - kWave) {   // the last wave, which has the fewest keys
    const double z0 = soft_lse(soft_reduce<false>(st));   // over 16 lanes, the same in each row of them
    if (tid == kJoinNT - 1) s_lse = z0;
  }
  __syncthreads();
  const double z0 = s_lse;
  int mine = 0, top_step = 1;
  while (2 * top_step <= K) top_step *= 2;
  for (int k = tid; k < parts * K; k += kJoinNT) {
    const uint64_t key = s_key[k];
    if (key == 0) continue;
    ++mine;
    int before[kMaxParts] = {};   // entries of each list that are above the key
    for (int step = top_step; step > 0; step /= 2) {   // all lists at a time: what is read is in LDS, and its latency counts
      uint64_t x[kMaxParts];
#pragma unroll
      for (int p = 0; p < kMaxParts; ++p) x[p] = s_key[min(p, parts - 1) * K + min(before[p] + step, K) - 1];
#pragma unroll
      for (int p = 0; p < kMaxParts; ++p) before[p] += before[p] + step <= K && x[p] > key ? step : 0;
    }
    int rank = 0;
#pragma unroll
    for (int p = 0; p < kMaxParts; ++p) rank += p < parts ? before[p] : 0;
    if (rank < K) {
      index[t * K + rank] = key_id(key);
      logprob[t * K + rank] = float(double(key_logit(key)) - z0);
    }
  }
  if (mine) atomicAdd(&s_n, mine);
  __syncthreads();
  for (int k = s_n + tid; k < K; k += kJoinNT) {
    index[t * K + k] = -1;
    logprob[t * K + k] = -INFINITY;
  }
  if (tid == 0 && lse) lse[t] = float(z0);
}

// Parts of a row: a workgroup per CU in all.  (151936 bf16, K = 64, one / two / four workgroups per CU: 64 rows 15.4 / 17.0 / 16.9 us,
// 200 17.5 / 24.7 / 26.0, 300 26.7 / 26.6 / 30.5.)
static int topk_parts(int64_t T, int nvec, int cus) {
  if (T > cus / 2 || nvec < 2 * 4 * 256) return 1;
  return int(std::min<int64_t>({kMaxParts, cus / T, nvec / (4 * 256)}));
}

size_t topk_workspace_bytes(int64_t T, int32_t V, int32_t K) {
  (void)V;
  const int64_t rows = std::min<int64_t>(T, compute_units());   // more are not split
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
  auto launch = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, grid, dim3(unsigned(threads)), 0, s, logits, V, ld, row_active, K, index, logprob, lse, keys, sums);
  };
  // Held / streaming by: bf16 K = 64, 64 rows of 2399 6.7 / 7.2 us, 4000 of 1024 17.6 / 23.2; fp32, 4000 of 2399 19.6 / 25.2.  Where rows queue,
  // waiting threads cost more than vectors in turn: 5000 rows of 14464 with 1024 / 256 threads 79 / 47 us, 40 rows 7.1 / 7.8.  Eight vectors held are
  // no gain: 5000 of 14464 49.6 / 47.3.  More than 128 of 256 maxima would be no threshold.  151936, streaming by 512 / 1024: 200 rows, K = 16, 64,
  // 256: 16.8 / 16.5, 18.0 / 17.5, 21.2 / 20.1 us; 300 rows 26.7 / 28.8, 4096 203 / 214 at K = 64.
  const bool many = T > 2 * compute_units();
  if (K <= 128 && per <= 2 * 256) launch(k_topk<256, DT, VEC, 2>, 256);
  else if (K <= 128 && per <= 4 * 256 && many) launch(k_topk<256, DT, VEC, 4>, 256);
  else if (per <= 2 * 512) launch(k_topk<512, DT, VEC, 2>, 512);
  else if (per <= 2 * 1024 && !many) launch(k_topk<1024, DT, VEC, 2>, 1024);
  else if (K <= 128 && per <= 4096 && many) launch(k_topk<256, DT, VEC, 0>, 256);
  else if (T * parts <= compute_units() && (parts == 1 || K > 128)) launch(k_topk<1024, DT, VEC, 0>, 1024);
  else launch(k_topk<512, DT, VEC, 0>, 512);
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
  // Element by element where a row has few vectors for K: their maxima hardly make a threshold (64 rows of 2399, K = 256: 20 us for 255)
  const bool vec = rows_alike(logits, nullptr, storage_bytes(dtype)) && int64_t(V) * storage_bytes(dtype) / 16 >= 2 * K;
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
