// Embedding rows looked up and scaled, and the gradient of the table from tokens sorted by id.
//
// The sort is a launch of independent workgroups, each of which owns the ids that are alike modulo their number: it counts
// its own ids one by one and the tokens of those in front of it as a whole, and places its tokens in ascending order within an id.
// Every token is read by every workgroup, out of the caches; nothing passes between workgroups and there are no counters whose order
// could show.  The sums are a second launch of workgroups that go over two kinds of work, found by halving in the owners' counts:
// pieces of kPiece tokens of frequent ids by column blocks, and whole rows of the others; and of small workgroups that zero the rows of the ids
// that no token has, 16 bytes a thread in the order of their addresses: that writes 6.5 TB/s, workgroups that walk over rows 5.2.
// Ids with several pieces are joined in order in a third.
#include <algorithm>

#include "row_scan.h"

namespace aero {

// One workgroup per token row.  VEC: rows of a vector and more, at any alignment; the last vector ends where the row ends and overlaps the one in
// front.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void k_embed_fwd(const void* __restrict__ table, int V, int H, const int32_t* __restrict__ ids,
                                                   float scale, void* __restrict__ out, int64_t ld_out,
                                                   int32_t* __restrict__ err_flag) {
  constexpr int E = VEC ? Storage<DT>::kPerVec : 1;
  const int64_t t = blockIdx.x;
  const int id = ids[t];
  if (id >= V && threadIdx.x == 0 && err_flag) atomicOr(err_flag, AERO_DERR_BAD_TARGET);
  const bool there = id >= 0 && id < V;
  for (int c0 = threadIdx.x * E; c0 < H; c0 += 256 * E) {
    const int c = min(c0, H - E);
    const char* const src = row_ptr<DT>(table, there ? id : 0, H, c);
    char* const dst = row_ptr<DT>(out, t, ld_out, c);
    if constexpr (VEC) {
      u32x4_t v = {0u, 0u, 0u, 0u};
      if (there) {
        float x[E];
        const u32x4_t in = *reinterpret_cast<const u32x4_any_t*>(src);
        unpack_vec<DT>(in, x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] *= scale;
        v = pack_vec<DT>(x);
      }
      *reinterpret_cast<u32x4_any_t*>(dst) = v;
    } else {
      store_elt<DT>(dst, 0, there ? scale * load_elt<DT>(src, 0) : 0.f);
    }
  }
}

// ---- gradient ----
constexpr int kSortNT = 1024, kSortWaves = kSortNT / kWave;
constexpr int kSortRuns = 8, kSortEach = 4, kSortRun = kSortNT * kSortEach, kSortChunk = kSortRun * kSortRuns;   // tokens that a sorting workgroup holds
constexpr int kListed = 16384;                           // of its own among them that it places at a time
constexpr int kLogBins = 10, kBins = 1 << kLogBins;      // ids of a sorting workgroup
constexpr int kMinOwners = 256;                          // sorting workgroups, a power of two
constexpr int kPiece = 32;                               // tokens of a frequent id that one wave adds up
constexpr int kFew = 4;                                  // up to so many tokens: a wave takes the whole row

// Sorted tokens [start, start + count) of an id.  row: where the sum goes when the id has several pieces, -1: to the table.
struct Piece {
  int32_t id, start, count, row;
};
// An id with several pieces, whose sums are rows [row, row + pieces).
struct Whole {
  int32_t id, row, pieces, pad;
};
// How many of each a sorting workgroup has.  Its pieces lie from its first sorted position on: those of frequent ids in front, the
// others behind, from the last position backwards; its wholes from the same position on.
struct OwnerCounts {
  int32_t *heavy, *few, *whole;   // [owners]
  int32_t *base, *end;            // [owners] first sorted position, and the one behind the last
};

static int embed_owners(int32_t V) {
  int owners = kMinOwners;
  while (int64_t(owners) * kBins < V) owners *= 2;
  return owners;
}
struct EmbedWorkspace {
  int32_t* order;   // [T] tokens sorted by id
  Piece* piece;     // [T]
  Whole* whole;     // [T]
  uint8_t* there;   // [V] a token has the id
  OwnerCounts n;
  float* partial;   // [2 (T / kPiece + 1)][H]
  size_t bytes;
};
static EmbedWorkspace embed_workspace(void* base, int64_t T, int32_t V, int64_t H) {
  char* const p = reinterpret_cast<char*>(base);
  size_t at = 0;
  auto take = [&](size_t n) {
    char* const q = p + at;
    at += (n + 255) / 256 * 256;
    return q;
  };
  const size_t owners = embed_owners(V);
  EmbedWorkspace w;
  w.order = reinterpret_cast<int32_t*>(take(size_t(T) * 4));
  w.piece = reinterpret_cast<Piece*>(take(size_t(T) * sizeof(Piece)));
  w.whole = reinterpret_cast<Whole*>(take(size_t(T) * sizeof(Whole)));
  w.there = reinterpret_cast<uint8_t*>(take(size_t(V)));
  int32_t** const counts[] = {&w.n.heavy, &w.n.few, &w.n.whole, &w.n.base, &w.n.end};
  for (int32_t** c : counts) *c = reinterpret_cast<int32_t*>(take(owners * 4));
  w.partial = reinterpret_cast<float*>(take(size_t(2 * (T / kPiece + 1)) * size_t(H) * 4));
  w.bytes = at + 256;
  return w;
}
size_t embedding_workspace_bytes(int64_t T, int32_t V, int32_t H) {
  return embed_workspace(nullptr, T, V > 0 ? V : 1, H > 0 ? H : 0).bytes;
}

// Workgroup g owns the ids with id % owners == g.  A chunk of tokens is kSortRuns runs, of which a thread holds kSortEach tokens that follow
// each other: (run, thread, number) is their order.
__global__ __launch_bounds__(kSortNT) void k_embed_sort(const int32_t* __restrict__ ids, int64_t T, int V, int log_owners,
                                                        int32_t* __restrict__ order, Piece* __restrict__ pieces, Whole* __restrict__ wholes,
                                                        uint8_t* __restrict__ there, OwnerCounts counts, int32_t* __restrict__ err_flag) {
  __shared__ int s_count[kBins], s_at[kBins];
  __shared__ int s_wave[2][kSortWaves], s_run[kSortRuns * kSortWaves], s_all;
  __shared__ int s_n[3];
  __shared__ uint32_t s_list[kListed];                // own tokens in order: place in the chunk << kLogBins | id
  static_assert(uint64_t(kSortChunk) << kLogBins <= uint64_t(1) << 32 && kListed < 1 << 16, "a word each; counts of half a word");
  __shared__ uint32_t s_seg[kSortWaves][kBins / 2];   // listed tokens of an id in a wave's segment; ids 2 k and 2 k + 1 share a word
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = blockIdx.x, mask = (1 << log_owners) - 1;
  const int bins = (V - g + mask) >> log_owners;   // ids g, g + owners, ... below V
  const uint64_t below = (uint64_t(1) << lane) - 1;
  s_count[tid] = 0;
  if (tid < 3) s_n[tid] = 0;
  __syncthreads();
  // ---- count ----
  int id[kSortRuns][kSortEach];
  uint32_t own = 0;   // bit kSortEach r + u: id[r][u] is this workgroup's
  int before = 0;
  bool bad = false;
  auto load = [&](int64_t t0, bool count) {
    const bool whole = t0 + kSortChunk <= T && reinterpret_cast<uintptr_t>(ids) % 16 == 0;   // uniform
#pragma unroll
    for (int r = 0; r < kSortRuns; ++r) {
      const int64_t t = t0 + r * kSortRun + tid * kSortEach;
      if (whole) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(ids + t);
        id[r][0] = int(v.x); id[r][1] = int(v.y); id[r][2] = int(v.z); id[r][3] = int(v.w);
      } else {
#pragma unroll
        for (int u = 0; u < kSortEach; ++u) id[r][u] = t + u < T ? ids[t + u] : -1;
      }
    }
    own = 0;
#pragma unroll
    for (int r = 0; r < kSortRuns; ++r) {
      if (t0 + r * kSortRun >= T) break;   // uniform
#pragma unroll
      for (int u = 0; u < kSortEach; ++u) {
        const int i = id[r][u], owner = uint32_t(i) < uint32_t(V) ? i & mask : kSortNT * kBins;
        own |= owner == g ? 1u << (kSortEach * r + u) : 0u;
        if (count) {
          before += owner < g;
          bad |= i >= V;
          if (owner == g) atomicAdd(&s_count[i >> log_owners], 1);
        }
      }
    }
  };
  for (int64_t t0 = 0; t0 < T; t0 += kSortChunk) load(t0, true);
  if (g == 0 && bad && err_flag) atomicOr(err_flag, AERO_DERR_BAD_TARGET);
  before = wave_sum_i(before);
  if (lane == 0) s_wave[0][wave] = before;
  __syncthreads();
  // ---- where each id starts ----
  static_assert(kBins == kSortNT, "a thread per id");
  const int mine = s_count[tid];
  int incl = mine;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int y = __shfl_up(incl, m, kWave);
    if (lane >= m) incl += y;
  }
  if (lane == kWave - 1) s_wave[1][wave] = incl;
  __syncthreads();
  int base = 0, start = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    base += s_wave[0][w];
    if (w < wave) start += s_wave[1][w];
    total += s_wave[1][w];
  }
  start += base;
  s_at[tid] = start;
  // ---- pieces, in whatever order ----
  const int id_mine = (tid << log_owners) + g;
  if (tid < bins) there[id_mine] = mine > 0;
  const int np = mine > kFew ? (mine + kPiece - 1) / kPiece : 0;
  const int row = 2 * (start / kPiece);   // np <= 2 (mine / kPiece): the next id's rows lie behind
  int at = 0;
  if (mine > kFew) {
    at = base + atomicAdd(&s_n[0], np);
    if (np > 1) wholes[base + atomicAdd(&s_n[2], 1)] = Whole{id_mine, row, np, 0};
    else pieces[at] = Piece{id_mine, start, mine, -1};
  } else if (mine > 0) {
    pieces[base + total - 1 - atomicAdd(&s_n[1], 1)] = Piece{id_mine, start, mine, -1};
  }
  for (uint64_t m = __builtin_amdgcn_ballot_w64(np > 1); m != 0; m &= m - 1) {   // several pieces: by all lanes (one lane, 1024 of them: 45 us)
    const int l = __builtin_ctzll(m);
    const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
    for (int k = lane; k < of(np); k += kWave)
      pieces[of(at) + k] = Piece{of(id_mine), of(start) + k * kPiece, min(kPiece, of(mine) - k * kPiece), of(row) + k};
  }
  __syncthreads();
  if (tid == 0) {
    counts.heavy[g] = s_n[0];
    counts.few[g] = s_n[1];
    counts.whole[g] = s_n[2];
    counts.base[g] = base;
    counts.end[g] = base + total;
  }
  // ---- place, in order ----
  if (total == 0) return;
  for (int64_t t0 = 0; t0 < T; t0 += kSortChunk) {
    if (T > kSortChunk) load(t0, false);   // a single chunk is still there
    // own tokens of the run in the lanes in front, and in the wave: three runs to a word (a wave has 256 tokens of a run)
    int ahead[kSortRuns];
#pragma unroll
    for (int r0 = 0; r0 < kSortRuns; r0 += 3) {
      uint32_t mine3 = 0;
#pragma unroll
      for (int r = r0; r < kSortRuns && r < r0 + 3; ++r) mine3 |= uint32_t(__popc(own >> (kSortEach * r) & ((1u << kSortEach) - 1))) << (10 * (r - r0));
      const uint32_t up_to = wave_scan(mine3);
#pragma unroll
      for (int r = r0; r < kSortRuns && r < r0 + 3; ++r) {
        ahead[r] = int((up_to - mine3) >> (10 * (r - r0)) & 1023);
        if (lane == kWave - 1) s_run[r * kSortWaves + wave] = int(up_to >> (10 * (r - r0)) & 1023);
      }
    }
    __syncthreads();
    static_assert(kSortRuns * kSortWaves == 2 * kWave, "two counts per lane");
    if (wave == 0) {
      const int x = s_run[2 * lane], y = s_run[2 * lane + 1];
      int sum = x + y;
#pragma unroll
      for (int m = 1; m < kWave; m <<= 1) {
        const int z = __shfl_up(sum, m, kWave);
        if (lane >= m) sum += z;
      }
      s_run[2 * lane] = sum - x - y;
      s_run[2 * lane + 1] = sum - y;
      if (lane == kWave - 1) s_all = sum;
    }
    __syncthreads();
    const int n = s_all;
    for (int from = 0; from < n; from += kListed) {   // kListed of the workgroup's own tokens at a time
      if (own != 0) {
#pragma unroll
        for (int r = 0; r < kSortRuns; ++r) {
          if ((own >> (kSortEach * r) & ((1u << kSortEach) - 1)) == 0) continue;
          int at = s_run[r * kSortWaves + wave] + ahead[r] - from;
#pragma unroll
          for (int u = 0; u < kSortEach; ++u) {
            if (own >> (kSortEach * r + u) & 1) {
              if (at >= 0 && at < kListed)
                s_list[at] = uint32_t(r * kSortRun + tid * kSortEach + u) << kLogBins | uint32_t(id[r][u] >> log_owners);
              ++at;
            }
          }
        }
      }
      __syncthreads();
      // 64 at a time: a token's place is its id's next one plus the lanes in front with the same id
      const int listed = min(n - from, kListed);
      auto same_id = [&](int k, int end, int& bin, int32_t& token) {   // lanes with the id of token k
        const bool in = k < end;
        const uint32_t x = in ? s_list[k] : 0;
        bin = int(x & (kBins - 1));
        token = int32_t(t0 + (x >> kLogBins));
        uint64_t same = __builtin_amdgcn_ballot_w64(in);
#pragma unroll
        for (int bit = 0; bit < kLogBins; ++bit) {
          const uint64_t m = __builtin_amdgcn_ballot_w64((bin >> bit & 1) != 0);
          same &= (bin >> bit & 1) != 0 ? m : ~m;
        }
        return same;
      };
      if (listed <= kWave) {
        if (wave == 0) {
          int bin, token;
          const uint64_t same = same_id(lane, listed, bin, token);
          if (lane < listed) {
            const int rank = __popcll(same & below), at = s_at[bin];
            order[at + rank] = token;
            if (rank == 0) s_at[bin] = at + __popcll(same);   // behind the read by every lane of the id: one wave, in step
          }
        }
      } else {
        // A segment of the list to each wave, which counts its ids; a thread per two ids turns the counts into offsets.  (All by one wave:
        // 253 us for 32768 tokens of one id, 28 instead of 19 for ids whose frequency falls as 1 / rank.)
        const int each = (listed + kSortNT - 1) / kSortNT * kWave, segs = (listed + each - 1) / each;
        const int k0 = wave * each, k1 = min(k0 + each, listed);
        if (wave < segs) {
#pragma unroll
          for (int k = 0; k < kBins / 2 / kWave; ++k) s_seg[wave][k * kWave + lane] = 0;
          __builtin_amdgcn_wave_barrier();
          for (int k = k0 + lane; k < k1; k += kWave) {
            const uint32_t bin = s_list[k] & (kBins - 1);
            atomicAdd(&s_seg[wave][bin / 2], bin % 2 ? 0x10000u : 1u);
          }
        }
        __syncthreads();
        uint32_t up_to = 0;
        if (tid < kBins / 2)
          for (int w = 0; w < segs; ++w) {
            const uint32_t x = s_seg[w][tid];
            s_seg[w][tid] = up_to;
            up_to += x;   // at most kListed in either half
          }
        __syncthreads();
        for (int k = k0; k < k1; k += kWave) {
          int bin, token;
          const uint64_t same = same_id(k + lane, k1, bin, token);
          if (k + lane < k1) {
            const int rank = __popcll(same & below), shift = bin % 2 * 16;
            const uint32_t offset = s_seg[wave][bin / 2] >> shift & 0xffffu;
            order[s_at[bin] + int(offset) + rank] = token;
            __builtin_amdgcn_wave_barrier();   // behind the read by every lane of the word
            if (rank == 0) atomicAdd(&s_seg[wave][bin / 2], uint32_t(__popcll(same)) << shift);
          }
          __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        if (tid < kBins / 2) {
          s_at[2 * tid] += int(up_to & 0xffffu);
          s_at[2 * tid + 1] += int(up_to >> 16);
        }
      }
      __syncthreads();
    }
    __syncthreads();
  }
}

// Inclusive sums of the owners' counts in LDS, and the owner that the u-th of all lies with (and which of its own it is).
constexpr int kSumNT = 256, kSumWaves = kSumNT / kWave;
__device__ __forceinline__ int scan_owners(const int32_t* __restrict__ n, int owners, int* s_end /*[owners]*/, int* s_wave /*[kSumWaves]*/) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  int total = 0;
  __syncthreads();   // s_end may still be in use
  for (int g0 = 0; g0 < owners; g0 += kSumNT) {   // owners is a multiple of kSumNT
    int incl = n[g0 + tid];
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
      const int y = __shfl_up(incl, m, kWave);
      if (lane >= m) incl += y;
    }
    if (lane == kWave - 1) s_wave[wave] = incl;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kSumWaves; ++w) {
      if (w < wave) incl += s_wave[w];
      all += s_wave[w];
    }
    s_end[g0 + tid] = total + incl;
    total += all;
    __syncthreads();
  }
  return total;
}
__device__ __forceinline__ int find_owner(const int* s_end, int owners, int u, int& own) {
  int lo = 0, hi = owners - 1;   // the first owner whose end is behind u
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (s_end[mid] > u) hi = mid;
    else lo = mid + 1;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  own = u - (lo > 0 ? __builtin_amdgcn_readfirstlane(s_end[lo - 1]) : 0);
  return lo;
}

// N sums, scaled, to consecutive columns of the table from the skip-th on: added to what is there, or in its place.
template <int OUT, int N> __device__ __forceinline__ void put_sums(char* at, const float (&sum)[N], int skip, float scale, bool accumulate) {
  float x[N];
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = scale * sum[e];
  if constexpr (N == Storage<OUT>::kPerVec) {
    if (skip == 0) {
      u32x4_any_t* const p = reinterpret_cast<u32x4_any_t*>(at);
      if (accumulate) {
        float y[N];
        const u32x4_t old = *p;
        unpack_vec<OUT>(old, y);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] += y[e];
      }
      const u32x4_any_t v = pack_vec<OUT>(x);
      __builtin_nontemporal_store(v, p);
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e >= skip) store_elt<OUT>(at, e, accumulate ? load_elt<OUT>(at, e) + x[e] : x[e]);
}

struct EmbedSums {
  const void* dout;
  int64_t ld;
  int H, owners;
  const int32_t* order;
  const Piece* piece;
  const uint8_t* there;
  OwnerCounts n;
  float scale;
  int accumulate;
  double per_width;      // 1 / H
  int V, workers;        // workgroups that go over the sums; others zero the table in the order of its addresses
  uint64_t zeros_from;   // the first of those
  float* partial;
  void* table;
};
// Sums of a lane: a 16-byte vector of the table (VEC: rows of one and more, at any alignment), so that a wave's stores follow each other (two
// vectors of fp32 from one of 16 bits, stored 32 bytes apart: 2 TB/s).  The last vector ends where the row ends and overlaps the one in front; its
// first elements are that one's to store.
template <int DT, int OUT, bool VEC> struct ColumnSums {
  static constexpr int E = VEC ? Storage<OUT>::kPerVec : 1, kBlock = kWave * E;
  struct Raw {
    uint32_t w[(E * Storage<DT>::kBytes + 3) / 4];
  };
  // Column blocks of `rows` rows that are asked for at a time: at most 32 registers of them.
  static constexpr int blocks(int rows) {
    const int n = 32 / (rows * int(sizeof(Raw) / 4));
    return n < 1 ? 1 : n > 8 ? 8 : n;
  }
  __device__ __forceinline__ static int column(const EmbedSums& a, int c) { return min(c, a.H - E); }
  __device__ __forceinline__ static Raw load(const EmbedSums& a, int token, int c) {
    const char* const at = row_ptr<DT>(a.dout, token, a.ld, c);
    Raw r;
    if constexpr (!VEC) {
      r.w[0] = load_raw<DT>(at, 0);
    } else if constexpr (sizeof(Raw) == 8) {
      const u32x2_any_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_any_t*>(at));
      r.w[0] = v.x; r.w[1] = v.y;
    } else {
#pragma unroll
      for (int k = 0; k < int(sizeof(Raw)) / 16; ++k) {
        const u32x4_any_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any_t*>(at) + k);
        r.w[4 * k] = v.x; r.w[4 * k + 1] = v.y; r.w[4 * k + 2] = v.z; r.w[4 * k + 3] = v.w;
      }
    }
    return r;
  }
  __device__ __forceinline__ static float elt(const Raw& r, int e) {
    if constexpr (Storage<DT>::kBytes == 4) return __uint_as_float(r.w[e]);
    else return widen<DT>(e % 2 ? r.w[e / 2] >> 16 : r.w[e / 2] & 0xffffu);
  }
  // R rows, of which `count` are there, C column blocks, all asked for before any is used
  template <int R, int C>
  __device__ __forceinline__ static void add(const EmbedSums& a, const int (&token)[R], int count, int c0, float (&sum)[C][E]) {
    Raw v[C][R];
#pragma unroll
    for (int b = 0; b < C; ++b)
#pragma unroll
      for (int k = 0; k < R; ++k) v[b][k] = load(a, token[k], column(a, c0 + b * kBlock));
#pragma unroll
    for (int b = 0; b < C; ++b)
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (k < count) {   // uniform
#pragma unroll
          for (int e = 0; e < E; ++e) sum[b][e] += elt(v[b][k], e);
        }
  }
  __device__ __forceinline__ static void put(const EmbedSums& a, int64_t id, int c, const float (&sum)[E]) {
    if (c >= a.H) return;
    const int at = column(a, c);
    put_sums<OUT, E>(row_ptr<OUT>(a.table, id, a.H, at), sum, c - at, a.scale, a.accumulate != 0);
  }
  // the whole row of an id with R tokens
  template <int R, int C> __device__ __forceinline__ static void row(const EmbedSums& a, const Piece& p, int own) {
    int token[R];
#pragma unroll
    for (int k = 0; k < R; ++k) token[k] = __builtin_amdgcn_readlane(own, k);
    for (int c0 = threadIdx.x % kWave * E; c0 < a.H; c0 += C * kBlock) {
      float sum[C][E] = {};
      add<R, C>(a, token, R, c0, sum);
#pragma unroll
      for (int b = 0; b < C; ++b) put(a, p.id, c0 + b * kBlock, sum[b]);
    }
  }
};

// A vector of the table by each thread of the workgroup, from element `before` on: zeros where no token has the row's id.  A vector that spans
// two rows is stored whole where both are empty, and otherwise element by element.
template <int OUT> __device__ __forceinline__ void put_zeros(const EmbedSums& a, uint64_t before) {
  constexpr int Z = Storage<OUT>::kPerVec;
  const uint32_t H = uint32_t(a.H);
  const uint64_t all = uint64_t(a.V) * H, from = before + threadIdx.x * Z;
  if (from >= all) return;
  char* const at = reinterpret_cast<char*>(a.table) + from * Storage<OUT>::kBytes;
  // row and column of the vector, by reciprocals and a correction (whole-number division: a third of the time of a narrow table)
  uint32_t base = uint32_t(double(before) * a.per_width);
  int64_t rest = int64_t(before) - int64_t(uint64_t(base) * H);
  if (rest < 0) rest += H, --base;
  if (rest >= int64_t(H)) rest -= H, ++base;
  const uint32_t in = uint32_t(rest) + threadIdx.x * Z;
  uint32_t more = uint32_t(float(in) * float(a.per_width));
  int32_t column = int32_t(in - more * H);
  if (column < 0) column += H, --more;
  if (column >= int32_t(H)) column -= H, ++more;
  const uint32_t row = base + more, left = H - uint32_t(column);   // columns of the row from here on
  const bool spans = left < Z;
  const bool none = !a.there[row], next_none = !a.there[min(row + 1, uint32_t(a.V) - 1)];   // asked for together
  if (none && (!spans || (next_none && H >= Z && from + Z <= all))) {
    const u32x4_any_t zero = {0u, 0u, 0u, 0u};
    __builtin_nontemporal_store(zero, reinterpret_cast<u32x4_any_t*>(at));
  } else if (spans) {
#pragma unroll
    for (int e = 0; e < Z; ++e)
      if (from + e < all && (e < int(left) ? none : H >= Z ? next_none : !a.there[row + 1 + (e - left) / H])) store_elt<OUT>(at, e, 0.f);
  }
}

// 80 registers, six workgroups to a CU: 16384 tokens of width 1536 in bf16, 69 us; eight workgroups, with registers spilled, 74; five, 71.
template <int DT, int OUT, bool VEC> __global__ __launch_bounds__(kSumNT, 6) void k_embed_sum(EmbedSums a) {
  using Sums = ColumnSums<DT, OUT, VEC>;
  constexpr int E = Sums::E, Z = Storage<OUT>::kPerVec;
  extern __shared__ int s_end[];   // [owners]
  __shared__ int s_wave[kSumWaves];
  const int lane = threadIdx.x % kWave;
  if (int(blockIdx.x) >= a.workers) {
    put_zeros<OUT>(a, (a.zeros_from + (blockIdx.x - uint32_t(a.workers))) * (kSumNT * Z));
    return;
  }
  const int first = __builtin_amdgcn_readfirstlane(int(blockIdx.x) * kSumWaves + int(threadIdx.x) / kWave), waves = a.workers * kSumWaves;
  // ---- pieces of frequent ids, by column blocks ----
  const int blocks = (a.H + Sums::kBlock - 1) / Sums::kBlock;
  int64_t units = int64_t(scan_owners(a.n.heavy, a.owners, s_end, s_wave)) * blocks;
  for (int64_t u = first; u < units; u += waves) {
    int k;
    const int g = find_owner(s_end, a.owners, int(u / blocks), k);
    const Piece p = a.piece[a.n.base[g] + k];
    const int own = lane < p.count ? a.order[p.start + lane] : 0;   // lane k: the piece's k-th token
    const int c = int(u % blocks) * Sums::kBlock + lane * E;
    float sum[1][E] = {};
    constexpr int R = sizeof(typename Sums::Raw) > 16 ? 4 : 8;
    for (int k0 = 0; k0 < p.count; k0 += R) {
      int token[R];
#pragma unroll
      for (int r = 0; r < R; ++r) token[r] = __builtin_amdgcn_readlane(own, min(k0 + r, p.count - 1));
      Sums::template add<R, 1>(a, token, p.count - k0, c, sum);
    }
    if (p.row < 0) {
      Sums::put(a, p.id, c, sum[0]);
    } else if (c < a.H) {   // columns that overlap have the same sums
#pragma unroll
      for (int e = 0; e < E; ++e) a.partial[size_t(p.row) * a.H + Sums::column(a, c) + e] = sum[0][e];
    }
  }
  // ---- whole rows of the others ----
  units = scan_owners(a.n.few, a.owners, s_end, s_wave);
  for (int64_t u = first; u < units; u += waves) {
    int k;
    const int g = find_owner(s_end, a.owners, int(u), k);
    const Piece p = a.piece[a.n.end[g] - 1 - k];
    const int own = lane < p.count ? a.order[p.start + lane] : 0;
    static_assert(kFew == 4, "cases below");
    switch (p.count) {   // uniform
      case 1: Sums::template row<1, Sums::blocks(1)>(a, p, own); break;
      case 2: Sums::template row<2, Sums::blocks(2)>(a, p, own); break;
      case 3: Sums::template row<3, Sums::blocks(3)>(a, p, own); break;
      default: Sums::template row<4, Sums::blocks(4)>(a, p, own);
    }
  }
}

// Ids with several pieces: workgroup by (id, kWave columns), a quarter of the pieces to each wave.
template <int OUT>
__global__ __launch_bounds__(kSumNT) void k_embed_join(EmbedSums a, const Whole* __restrict__ wholes) {
  extern __shared__ int s_end[];   // [owners]
  __shared__ int s_wave[kSumWaves];
  __shared__ float s_sum[kSumWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int blocks = (a.H + kWave - 1) / kWave;
  const int64_t units = int64_t(scan_owners(a.n.whole, a.owners, s_end, s_wave)) * blocks;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    int k;
    const int g = find_owner(s_end, a.owners, int(u / blocks), k);
    const Whole w = wholes[a.n.base[g] + k];
    const int c = int(u % blocks) * kWave + lane;
    const float* const x = a.partial + size_t(w.row) * a.H + min(c, a.H - 1);
    const int each = (w.pieces + kSumWaves - 1) / kSumWaves, last = min((wave + 1) * each, w.pieces);
    float sum = 0.f;
    for (int r = wave * each; r < last; r += 8) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[size_t(min(r + e, last - 1)) * a.H];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (r + e < last) sum += y[e];
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    static_assert(kSumWaves == 4, "sums of a column");
    const float all[1] = {(s_sum[0][lane] + s_sum[1][lane]) + (s_sum[2][lane] + s_sum[3][lane])};
    if (wave == 0 && c < a.H) put_sums<OUT, 1>(row_ptr<OUT>(a.table, w.id, a.H, c), all, 0, a.scale, a.accumulate != 0);
    __syncthreads();   // s_sum is free again
  }
}

struct EmbedArgs {
  const void* dout;
  int64_t T;
  int H;
  int64_t ld;
  const int32_t* ids;
  int V;
  float scale;
  void* table;
  int accumulate;
  int32_t* err_flag;
};

constexpr int kWorkers = 6;                       // to a CU: 16384 tokens of 1000 ids, width 3584, 4 / 6 / 8: 67.7 / 63.3 / 63.1 us
constexpr int64_t kMaxZeros = int64_t(1) << 23;   // workgroups of a launch: half of the threads that a grid may have
template <int DT, int OUT> static void embed_bwd_launch(const EmbedArgs& a, void* workspace, hipStream_t s) {
  const EmbedWorkspace w = embed_workspace(workspace, a.T, a.V, a.H);
  const int owners = embed_owners(a.V), log_owners = __builtin_ctz(unsigned(owners));
  hipLaunchKernelGGL(k_embed_sort, dim3(unsigned(owners)), dim3(kSortNT), 0, s, a.ids, a.T, a.V, log_owners, w.order, w.piece, w.whole,
                     w.there, w.n, a.err_flag);
  constexpr int E = Storage<OUT>::kPerVec;
  const bool vec = a.H >= E;
  const int workers = kWorkers * compute_units();
  const int64_t zeros = a.accumulate ? 0 : (int64_t(a.V) * a.H + int64_t(kSumNT) * E - 1) / (int64_t(kSumNT) * E);
  EmbedSums sums{a.dout, a.ld, a.H, owners, w.order, w.piece, w.there, w.n, a.scale, a.accumulate, 1.0 / a.H, a.V, workers, 0, w.partial, a.table};
  const auto sum = vec ? k_embed_sum<DT, OUT, true> : k_embed_sum<DT, OUT, false>;
  const size_t lds = size_t(owners) * 4;   // at most 64 KB
  hipLaunchKernelGGL(sum, dim3(unsigned(workers + std::min(zeros, kMaxZeros))), dim3(kSumNT), lds, s, sums);
  sums.workers = 0;
  for (int64_t from = kMaxZeros; from < zeros; from += kMaxZeros) {
    sums.zeros_from = uint64_t(from);
    hipLaunchKernelGGL(sum, dim3(unsigned(std::min(zeros - from, kMaxZeros))), dim3(kSumNT), lds, s, sums);
  }
  if (a.T > kPiece)
    hipLaunchKernelGGL(k_embed_join<OUT>, dim3(unsigned(4 * compute_units())), dim3(kSumNT), lds, s, sums, w.whole);
}

template <int DT>
static void embed_fwd_launch(const void* table, int V, int H, const int32_t* ids, int64_t T, float scale, void* out, int64_t ld_out,
                             int32_t* err_flag, hipStream_t s) {
  const bool vec = H >= Storage<DT>::kPerVec;
  const auto fwd = vec ? k_embed_fwd<DT, true> : k_embed_fwd<DT, false>;
  hipLaunchKernelGGL(fwd, dim3(unsigned(T)), dim3(256), 0, s, table, V, H, ids, scale, out, ld_out, err_flag);
}

constexpr int kMaxWidth = 1 << 20;

}  // namespace aero

extern "C" aero_status aero_embedding_fwd(const void* table, int32_t dtype, int32_t V, int32_t H, const int32_t* ids, int64_t T, float scale,
                                          void* out, int64_t ld_out, int32_t* err_flag, void* stream) {
  using namespace aero;
  if (T < 0 || V < 1 || V > (1 << 24) || H < 1 || H > kMaxWidth || ld_out < H || !grid_fits(T, 1024)) return AERO_ERR_SHAPE;
  if (dtype != AERO_F32 && dtype != AERO_BF16 && dtype != AERO_F16) return AERO_ERR_DTYPE;
  if (T == 0) return AERO_OK;
  if (!table || !ids || !out) return AERO_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(table) % storage_bytes(dtype) != 0 || reinterpret_cast<uintptr_t>(out) % storage_bytes(dtype) != 0)
    return AERO_ERR_ALIGN;
  const hipStream_t s = as_stream(stream);
  switch (dtype) {
    case AERO_BF16: embed_fwd_launch<kBF16>(table, V, H, ids, T, scale, out, ld_out, err_flag, s); break;
    case AERO_F16: embed_fwd_launch<kF16>(table, V, H, ids, T, scale, out, ld_out, err_flag, s); break;
    default: embed_fwd_launch<kF32>(table, V, H, ids, T, scale, out, ld_out, err_flag, s);
  }
  return launch_status();
}

extern "C" aero_status aero_embedding_bwd(const void* dout, int32_t dtype, int64_t T, int32_t H, int64_t ld_dout, const int32_t* ids,
                                          int32_t V, float scale, void* dtable, int32_t dtable_dtype, int32_t* err_flag,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (T < 0 || V < 1 || V > (1 << 24) || H < 1 || H > kMaxWidth || ld_dout < H || !grid_fits(T, 1024)) return AERO_ERR_SHAPE;
  if (dtype != AERO_F32 && dtype != AERO_BF16 && dtype != AERO_F16) return AERO_ERR_DTYPE;
  const int32_t out_dtype = dtable_dtype & ~AERO_DW_ACCUMULATE;
  if (out_dtype != AERO_F32 && out_dtype != AERO_BF16) return AERO_ERR_DTYPE;
  if (!dtable || (T > 0 && (!dout || !ids))) return AERO_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(dout) % storage_bytes(dtype) != 0 || reinterpret_cast<uintptr_t>(dtable) % storage_bytes(out_dtype) != 0)
    return AERO_ERR_ALIGN;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < embedding_workspace_bytes(T, V, H))
    return AERO_ERR_WORKSPACE;
  const hipStream_t s = as_stream(stream);
  const EmbedArgs a{dout, T, H, ld_dout, ids, V, scale, dtable, dtable_dtype != out_dtype, err_flag};
  const bool f32 = out_dtype == AERO_F32;
  switch (dtype) {
    case AERO_BF16: f32 ? embed_bwd_launch<kBF16, kF32>(a, workspace, s) : embed_bwd_launch<kBF16, kBF16>(a, workspace, s); break;
    case AERO_F16: f32 ? embed_bwd_launch<kF16, kF32>(a, workspace, s) : embed_bwd_launch<kF16, kBF16>(a, workspace, s); break;
    default: f32 ? embed_bwd_launch<kF32, kF32>(a, workspace, s) : embed_bwd_launch<kF32, kBF16>(a, workspace, s);
  }
  return launch_status();
}
