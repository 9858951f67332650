// Embedding rows looked up and scaled, and the gradient of the table from tokens sorted by id.
//
// The sort is a launch of independent workgroups, each of which owns the ids that are alike modulo their number: it counts
// its own ids one by one and the tokens of those in front of it as a whole, and places its tokens in ascending order within an id.
// Every token is read by every workgroup, out of the caches; nothing passes between workgroups and there are no counters whose order
// could show.  A sorted place holds its token and where its id's tokens start and how many they are, so that the sums, a second launch,
// take the places as they lie: the places of kPiece tokens of an id share the row's columns among them, each of which it sums over all of
// these tokens, and so every place has the same work, however often its id occurs.  Beside them small workgroups zero the rows of the ids
// that no token has, 16 bytes a thread in the order of their addresses: that writes 6.5 TB/s, workgroups that walk over rows 5.2.
// Ids with several pieces are joined in order in a third.  A few hundred tokens take one launch instead (k_embed_few).
//
// The lookup is bound by its bytes: 16384 rows of 1536 bf16 14.4 us (6.8 TB/s).  The gradient by the table's: 600 tokens, 151936 x 1536 bf16 76 us (6.1 TB/s,
// the sort's 7.4 and the join's 4.5 included), 32768 tokens, 32000 x 3584 fp32 149 us (4.6 TB/s: sort 17, sums and zeros 126, join 8.5); of a
// small table by three launches (600 tokens of 1000 x 64 15 us), or by one (97 of 2589 x 367 4.2).
#include <algorithm>

#include "row_scan.h"

namespace aero {

// scale * E elements from src on, or zeros.
template <int DT, int E> __device__ __forceinline__ void look_up(const char* src, bool there, float scale, char* dst) {
  if constexpr (E > 1) {
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
// A workgroup per token row, or (NARROW) per `rows` of them, a thread a vector (32768 rows of 64 bf16: one a workgroup 9.0 us, 32 3.3; a row's
// address is scalar where it is the only one: 16384 rows of 1536 12.8 us for 13.5).  VEC: rows of a vector and more, at any alignment; the last
// vector ends where the row ends and overlaps the one in front.
constexpr int kLookNT = 256;
template <int DT, bool VEC, bool NARROW>
__global__ __launch_bounds__(kLookNT) void k_embed_fwd(const void* __restrict__ table, int V, int H, const int32_t* __restrict__ ids, int64_t T,
                                                       int rows, float scale, void* __restrict__ out, int64_t ld_out,
                                                       int32_t* __restrict__ err_flag) {
  constexpr int E = VEC ? Storage<DT>::kPerVec : 1;
  const uint32_t per = uint32_t(H + E - 1) / E, r = NARROW ? threadIdx.x / per : 0;
  const int64_t t = NARROW ? int64_t(blockIdx.x) * rows + r : blockIdx.x;
  if (NARROW && (r >= uint32_t(rows) || t >= T)) return;
  const int first = int((threadIdx.x - r * per) * E), id = ids[t];
  if (id >= V && first == 0 && err_flag) atomicOr(err_flag, AERO_DERR_BAD_TARGET);
  const bool there = id >= 0 && id < V;
  for (int c0 = first; c0 < H; c0 += kLookNT * E) {   // one turn where NARROW
    const int c = min(c0, H - E);
    look_up<DT, E>(row_ptr<DT>(table, there ? id : 0, H, c), there, scale, row_ptr<DT>(out, t, ld_out, c));
  }
}

// ---- gradient ----
constexpr int kSortNT = 1024, kSortWaves = kSortNT / kWave;
constexpr int kSortRuns = 8, kSortEach = 4, kSortRun = kSortNT * kSortEach, kSortChunk = kSortRun * kSortRuns;   // tokens that a sorting workgroup holds
constexpr int kListed = 16384;                           // of its own among them that it places at a time
constexpr int kLogBins = 10, kBins = 1 << kLogBins;      // ids of a sorting workgroup
constexpr int kMinOwners = 256;                          // sorting workgroups, a power of two
constexpr int kPiece = 32;                               // tokens of an id that are added up at a time
constexpr int kFew = 4;                                  // up to so many: several column blocks of a wave at a time

// A sorted place: a token, and its id's places [start, start + count).
struct Sorted {
  int32_t token, id, start, count;
};

static int embed_owners(int32_t V) {
  int owners = kMinOwners;
  while (int64_t(owners) * kBins < V) owners *= 2;
  return owners;
}
// First of the rows of partial sums of an id with several pieces; pieces <= 2 (count / kPiece), so that the next id's rows lie behind.
__host__ __device__ constexpr int piece_row(int start) { return 2 * (start / kPiece); }

struct EmbedWorkspace {
  Sorted* sorted;   // [T]
  int32_t* n;       // places that are taken
  uint8_t* there;   // [V] a token has the id
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
  EmbedWorkspace w;
  w.sorted = reinterpret_cast<Sorted*>(take(size_t(T) * sizeof(Sorted)));
  w.n = reinterpret_cast<int32_t*>(take(4));
  w.there = reinterpret_cast<uint8_t*>(take(size_t(V)));
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
                                                        Sorted* __restrict__ sorted, int32_t* __restrict__ n_sorted,
                                                        uint8_t* __restrict__ there, int32_t* __restrict__ err_flag) {
  __shared__ int s_count[kBins], s_start[kBins], s_at[kBins];   // an id's tokens, their first place, the next one's
  __shared__ int s_wave[2][kSortWaves], s_run[kSortRuns * kSortWaves], s_all;
  __shared__ uint32_t s_list[kListed];                // own tokens in order: place in the chunk << kLogBins | id
  static_assert(uint64_t(kSortChunk) << kLogBins <= uint64_t(1) << 32 && kListed < 1 << 16, "a word each; counts of half a word");
  __shared__ uint32_t s_seg[kSortWaves][kBins / 2];   // listed tokens of an id in a wave's segment; ids 2 k and 2 k + 1 share a word
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = blockIdx.x, mask = (1 << log_owners) - 1;
  const int bins = (V - g + mask) >> log_owners;   // ids g, g + owners, ... below V
  const uint64_t below = (uint64_t(1) << lane) - 1;
  s_count[tid] = 0;
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
  const int incl = int(wave_scan(uint32_t(mine)));
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
  s_start[tid] = start;
  s_at[tid] = start;
  if (tid < bins) there[(tid << log_owners) + g] = mine > 0;
  if (tid == 0 && g == mask) *n_sorted = base + total;
  __syncthreads();
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
      const int sum = int(wave_scan(uint32_t(x + y)));
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
      auto put = [&](int place, int token, int bin) {
        const u32x4_t x = {uint32_t(token), uint32_t((bin << log_owners) + g), uint32_t(s_start[bin]), uint32_t(s_count[bin])};
        reinterpret_cast<u32x4_t*>(sorted)[place] = x;
      };
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
            put(at + rank, token, bin);
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
            put(s_at[bin] + int(offset) + rank, token, bin);
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

constexpr int kSumNT = 256, kSumWaves = kSumNT / kWave;
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
  int H;
  const Sorted* sorted;
  const int32_t* n;
  const uint8_t* there;
  float scale;
  int accumulate;
  double per_width;      // 1 / H
  int V, workers;        // workgroups that go over the sums; others zero the table in the order of its addresses
  int log_split;         // waves that a place's columns are split over
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
  // Column blocks of `rows` rows that are asked for at a time: at most 24 registers of them.
  static constexpr int blocks(int rows) {
    const int n = 24 / (rows * int(sizeof(Raw) / 4));
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
  // R rows, of which `count` are there, C column blocks from c0 on, up to column `last`, all asked for before any is used
  template <int R, int C>
  __device__ __forceinline__ static void add(const EmbedSums& a, const int (&token)[R], int count, int c0, int last, float (&sum)[C][E]) {
    Raw v[C][R];
#pragma unroll
    for (int b = 0; b < C; ++b)
#pragma unroll
      for (int k = 0; k < R; ++k) v[b][k] = load(a, token[k], min(c0 + b * kBlock, last));
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
  // a row of the joined sums
  __device__ __forceinline__ static void keep(const EmbedSums& a, int row, int c, const float (&sum)[E]) {
    if (c >= a.H) return;
#pragma unroll
    for (int e = 0; e < E; ++e) a.partial[size_t(row) * a.H + column(a, c) + e] = sum[e];   // columns that overlap have the same sums
  }
  // column blocks [block, end) of an id with R tokens
  template <int R, int C> __device__ __forceinline__ static void columns(const EmbedSums& a, int id, int own, int block, int end) {
    int token[R];
#pragma unroll
    for (int k = 0; k < R; ++k) token[k] = __builtin_amdgcn_readlane(own, k);
    const int lane = threadIdx.x % kWave * E, last = column(a, (end - 1) * kBlock + lane);
    for (; block < end; block += C) {   // uniform
      float sum[C][E] = {};
      add<R, C>(a, token, R, block * kBlock + lane, last, sum);
#pragma unroll
      for (int b = 0; b < C; ++b)
        if (block + b < end) put(a, id, (block + b) * kBlock + lane, sum[b]);
    }
  }
};

// The table's row with an element: by a reciprocal and a correction.
__device__ __forceinline__ uint32_t row_of(const EmbedSums& a, uint64_t element) {
  const uint32_t row = uint32_t(double(element) * a.per_width);
  const int64_t rest = int64_t(element) - int64_t(uint64_t(row) * uint32_t(a.H));
  return rest < 0 ? row - 1 : rest >= a.H ? row + 1 : row;
}
// A vector of the table by each thread of the workgroup, from element `before` on: zeros where no token has the row's id.  A vector that spans
// two rows is stored whole where both are empty, and otherwise element by element.  (Two or four vectors a thread: 600 tokens, 151936 x 1536 bf16
// 89 and 96 us for 76.)
template <int OUT> constexpr uint64_t kZeroElts = uint64_t(kSumNT) * Storage<OUT>::kPerVec;   // of a workgroup
template <int OUT, class There> __device__ __forceinline__ void put_zeros(const EmbedSums& a, uint64_t before, There there) {
  constexpr int Z = Storage<OUT>::kPerVec;
  const uint32_t H = uint32_t(a.H);
  const uint64_t all = uint64_t(a.V) * H, from = before + threadIdx.x * Z;
  if (from >= all) return;
  char* const at = reinterpret_cast<char*>(a.table) + from * Storage<OUT>::kBytes;
  const uint32_t base = row_of(a, before);
  const uint32_t in = uint32_t(before - uint64_t(base) * H) + threadIdx.x * Z;
  uint32_t more = uint32_t(float(in) * float(a.per_width));
  int32_t column = int32_t(in - more * H);
  if (column < 0) column += H, --more;
  if (column >= int32_t(H)) column -= H, ++more;
  const uint32_t row = base + more, left = H - uint32_t(column);   // columns of the row from here on
  const bool spans = left < Z;
  const bool none = !there(row), next_none = !there(min(row + 1, uint32_t(a.V) - 1));   // asked for together
  if (none && (!spans || (next_none && H >= Z && from + Z <= all))) {
    const u32x4_any_t zero = {0u, 0u, 0u, 0u};
    __builtin_nontemporal_store(zero, reinterpret_cast<u32x4_any_t*>(at));
  } else if (spans) {
#pragma unroll
    for (int e = 0; e < Z; ++e)
      if (from + e < all && (e < int(left) ? none : H >= Z ? next_none : !there(row + 1 + (e - left) / H))) store_elt<OUT>(at, e, 0.f);
  }
}

// 64 registers, eight workgroups to a CU.  (With 32 registers of column blocks, six: one token of 151936 x 1536 fp32 142 us instead of 136.)
template <int DT, int OUT, bool VEC> __global__ __launch_bounds__(kSumNT, 8) void k_embed_sum(EmbedSums a) {
  using Sums = ColumnSums<DT, OUT, VEC>;
  constexpr int E = Sums::E;
  const int lane = threadIdx.x % kWave;
  if (int(blockIdx.x) >= a.workers) {
    put_zeros<OUT>(a, (a.zeros_from + (blockIdx.x - uint32_t(a.workers))) * kZeroElts<OUT>, [&](uint32_t row) { return a.there[row] != 0; });
    return;
  }
  const int first = __builtin_amdgcn_readfirstlane(int(blockIdx.x) * kSumWaves + int(threadIdx.x) / kWave), waves = a.workers * kSumWaves;
  const int units = *a.n << a.log_split, blocks = (a.H + Sums::kBlock - 1) / Sums::kBlock;
  const auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  // a place's record and its piece's tokens are asked for one and two turns ahead
  const auto record = [&](int64_t u) { return u < units ? a.sorted[u >> a.log_split] : Sorted{0, 0, 0, 0}; };
  const auto first_of = [&](int64_t u, int start) { return (int(u >> a.log_split) - start) / kPiece * kPiece; };   // of the piece's, from the id's
  const auto tokens = [&](int64_t u, const Sorted& x) {   // lane r: the piece's r-th token
    const int k = first_of(u, x.start);
    return lane < min(x.count - k, kPiece) ? a.sorted[x.start + k + lane].token : 0;
  };
  Sorted next = record(first), after = record(int64_t(first) + waves);
  int own = tokens(first, next);
  for (int64_t u = first; u < units; u += waves) {
    const Sorted at{0, uniform(next.id), uniform(next.start), uniform(next.count)};
    const int own_next = tokens(u + waves, after);
    next = after;
    after = record(u + 2 * waves);
    const int k = first_of(u, at.start), place = int(u >> a.log_split) - at.start - k, count = min(at.count - k, kPiece);
    // the piece's column blocks are dealt out over its places and their waves, evenly spaced
    const int share = count << a.log_split, mine = place << a.log_split | (int(u) & ((1 << a.log_split) - 1));
    const int block = mine * blocks / share, end = (mine + 1) * blocks / share;
    static_assert(kFew == 4, "cases below");
    switch (at.count <= kPiece ? count : kPiece) {   // uniform; a short last piece goes with the others of its id
      case 1: Sums::template columns<1, Sums::blocks(1)>(a, at.id, own, block, end); break;
      case 2: Sums::template columns<2, Sums::blocks(2)>(a, at.id, own, block, end); break;
      case 3: Sums::template columns<3, Sums::blocks(3)>(a, at.id, own, block, end); break;
      case 4: Sums::template columns<4, Sums::blocks(4)>(a, at.id, own, block, end); break;
      default:
        for (int b = block; b < end; ++b) {   // uniform
          const int c = b * Sums::kBlock + lane * E;
          float sum[1][E] = {};
          constexpr int R = sizeof(typename Sums::Raw) > 16 ? 4 : 8;
          for (int k0 = 0; k0 < count; k0 += R) {
            int token[R];
#pragma unroll
            for (int r = 0; r < R; ++r) token[r] = __builtin_amdgcn_readlane(own, min(k0 + r, count - 1));
            Sums::template add<R, 1>(a, token, count - k0, c, a.H - E, sum);
          }
          if (at.count <= kPiece) Sums::put(a, at.id, c, sum[0]);
          else Sums::keep(a, piece_row(at.start) + k / kPiece, c, sum[0]);
        }
    }
    own = own_next;
  }
}

// Ids with several pieces: their places take turns at kWave columns, a workgroup at a place; a quarter of the pieces to each of its waves.
template <int OUT>
__global__ __launch_bounds__(kSumNT) void k_embed_join(EmbedSums a) {
  __shared__ float s_sum[kSumWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int n = *a.n;
  for (int64_t p0 = blockIdx.x; p0 < n; p0 += int64_t(kWave) * gridDim.x) {   // a place by each lane, the same ones in every wave
    const int64_t p = p0 + int64_t(lane) * gridDim.x;
    Sorted x{0, 0, 0, 0};
    if (p < n) x = a.sorted[p];
    for (uint64_t m = __builtin_amdgcn_ballot_w64(x.count > kPiece); m != 0; m &= m - 1) {   // uniform
      const int l = __builtin_ctzll(m);
      const int id = __builtin_amdgcn_readlane(x.id, l), start = __builtin_amdgcn_readlane(x.start, l), count = __builtin_amdgcn_readlane(x.count, l);
      const int pieces = (count + kPiece - 1) / kPiece, each = (pieces + kSumWaves - 1) / kSumWaves, last = min((wave + 1) * each, pieces);
      for (int64_t c0 = (p0 + int64_t(l) * gridDim.x - start) * kWave; c0 < a.H; c0 += int64_t(count) * kWave) {
        const int c = int(c0) + lane;
        const float* const from = a.partial + size_t(piece_row(start)) * a.H + min(c, a.H - 1);
        float sum = 0.f;
        for (int r = wave * each; r < last; r += 8) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = from[size_t(min(r + e, last - 1)) * a.H];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (r + e < last) sum += y[e];
        }
        s_sum[wave][lane] = sum;
        __syncthreads();
        static_assert(kSumWaves == 4, "sums of a column");
        const float all[1] = {(s_sum[0][lane] + s_sum[1][lane]) + (s_sum[2][lane] + s_sum[3][lane])};
        if (wave == 0 && c < a.H) put_sums<OUT, 1>(row_ptr<OUT>(a.table, id, a.H, c), all, 0, a.scale, a.accumulate != 0);
        __syncthreads();   // s_sum is free again
      }
    }
  }
}

// A few hundred tokens need no sort: one launch, in which a workgroup per token and column block sums up the tokens with its id, 64 to a wave in turn, if
// it is the first of them, and those that zero the table see from the ids whether one has a row of theirs.  Sorted / so: 97 tokens, 2589 x 367
// 13.2 / 4.2 us; 256 of 151936 x 1536 bf16 75 / 72; 500 of 20000 x 368 20 / 10.8.  Every zeroing wave reads the ids, so that more than 256 take it for
// tables of up to 64 MB only: 500 of 33 MB 21 / 13.5 us, of 123 MB 29.9 / 30.9, 300 of 467 MB 75 / 95.
constexpr int kFewWords = 4, kMoreWords = 8;   // of 64 tokens
constexpr int64_t kMoreZeros = 16384;          // workgroups
template <int DT, int OUT, bool VEC, int WORDS>
__global__ __launch_bounds__(kSumNT) void k_embed_few(EmbedSums a, const int32_t* __restrict__ ids, int T, int blocks, int32_t* __restrict__ err_flag) {
  using Sums = ColumnSums<DT, OUT, VEC>;
  constexpr int E = Sums::E;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  if (int(blockIdx.x) >= a.workers) {   // each wave by itself
    const uint64_t before = (a.zeros_from + (blockIdx.x - uint32_t(a.workers))) * kZeroElts<OUT>;
    const uint32_t r0 = row_of(a, before), r1 = row_of(a, before + kZeroElts<OUT> - 1);
    int own[WORDS];
    uint64_t meant[WORDS], any = 0;   // tokens with a row of the workgroup's
#pragma unroll
    for (int w = 0; w < WORDS; ++w) own[w] = w * kWave + lane < T ? ids[w * kWave + lane] : -1;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      meant[w] = __builtin_amdgcn_ballot_w64(own[w] >= 0 && uint32_t(own[w]) >= r0 && uint32_t(own[w]) <= r1);
      any |= meant[w];
    }
    if (any == 0) {   // uniform
      put_zeros<OUT>(a, before, [](uint32_t) { return false; });
    } else {
      put_zeros<OUT>(a, before, [&](uint32_t row) {
        bool yes = false;
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
          for (uint64_t m = meant[w]; m != 0;) {   // an id once
            const int one = __builtin_amdgcn_readlane(own[w], __builtin_ctzll(m));
            yes |= uint32_t(one) == row;
            m &= (m - 1) & ~__builtin_amdgcn_ballot_w64(own[w] == one);
          }
        return yes;
      });
    }
    return;
  }
  __shared__ uint64_t s_same[WORDS];
  __shared__ float s_sum[kSumWaves][E][kWave];
  const int t = int(blockIdx.x) / blocks, block = int(blockIdx.x) % blocks;
  const int own = ids[t];
  uint64_t same[WORDS / kSumWaves], mine = 0;   // tokens with the id, 64 in a word: the wave's are every fourth
#pragma unroll
  for (int k = 0; k < WORDS / kSumWaves; ++k) {
    const int w = k * kSumWaves + wave, id = w * kWave + lane < T ? ids[w * kWave + lane] : -1;
    if (blockIdx.x == 0 && id >= a.V && err_flag) atomicOr(err_flag, AERO_DERR_BAD_TARGET);
    same[k] = __builtin_amdgcn_ballot_w64(id == own);
    mine |= same[k];
    if (lane == 0) s_same[w] = same[k];
  }
  if (own < 0 || own >= a.V) return;   // uniform
  __syncthreads();
  bool has[kSumWaves] = {};   // waves with tokens of the id
#pragma unroll
  for (int w = 0; w < WORDS; ++w) {
    const uint64_t m = s_same[w], in_front = t / kWave > w ? ~uint64_t(0) : t / kWave == w ? (uint64_t(1) << (t % kWave)) - 1 : 0;
    if ((m & in_front) != 0) return;   // uniform: not the first
    has[w % kSumWaves] |= m != 0;
  }
  const int waves = has[0] + has[1] + has[2] + has[3];
  const int c = block * Sums::kBlock + lane * E;
  float sum[1][E] = {};
  constexpr int R = sizeof(typename Sums::Raw) > 16 ? 4 : sizeof(typename Sums::Raw) > 8 ? 8 : 16;
#pragma unroll
  for (int k = 0; k < WORDS / kSumWaves; ++k)
    for (uint64_t rest = same[k]; rest != 0;) {   // uniform in the wave; R tokens in ascending order
      int token[R], count = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (rest != 0) {
          token[r] = (k * kSumWaves + wave) * kWave + __builtin_ctzll(rest);
          rest &= rest - 1;
          ++count;
        } else {
          token[r] = token[0];
        }
      }
      Sums::template add<R, 1>(a, token, count, c, a.H - E, sum);
    }
  if (waves == 1) {   // uniform
    if (mine != 0) Sums::put(a, own, c, sum[0]);
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_sum[wave][e][lane] = sum[0][e];
  __syncthreads();
  if (wave != 0) return;
  static_assert(kSumWaves == 4, "sums of a column");
#pragma unroll
  for (int e = 0; e < E; ++e) sum[0][e] = (s_sum[0][e][lane] + s_sum[1][e][lane]) + (s_sum[2][e][lane] + s_sum[3][e][lane]);
  Sums::put(a, own, c, sum[0]);
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

constexpr int kWorkers = 8;                       // to a CU: 16384 tokens of 1000 ids, width 3584, 6 / 8 / 12: 62.4 / 56.1 / 57.7 us
constexpr int64_t kMaxZeros = int64_t(1) << 23;   // workgroups of a launch: half of the threads that a grid may have
template <int DT, int OUT> static void embed_bwd_launch(const EmbedArgs& a, void* workspace, hipStream_t s) {
  const EmbedWorkspace w = embed_workspace(workspace, a.T, a.V, a.H);
  constexpr int E = Storage<OUT>::kPerVec;
  const bool vec = a.H >= E;
  const int blocks = (a.H + kWave * (vec ? E : 1) - 1) / (kWave * (vec ? E : 1));
  const int64_t zeros = a.accumulate ? 0 : int64_t((uint64_t(a.V) * a.H + kZeroElts<OUT> - 1) / kZeroElts<OUT>);
  EmbedSums sums{a.dout, a.ld, a.H, w.sorted, w.n, w.there, a.scale, a.accumulate, 1.0 / a.H, a.V, 0, 0, 0, w.partial, a.table};
  const bool more = a.T > kFewWords * kWave;
  if (a.T <= kMoreWords * kWave && (!more || zeros <= kMoreZeros)) {
    const auto few = more ? (vec ? k_embed_few<DT, OUT, true, kMoreWords> : k_embed_few<DT, OUT, false, kMoreWords>)
                          : (vec ? k_embed_few<DT, OUT, true, kFewWords> : k_embed_few<DT, OUT, false, kFewWords>);
    sums.workers = int(a.T) * blocks;
    for (int64_t from = 0; from == 0 || from < zeros; from += kMaxZeros) {
      sums.zeros_from = uint64_t(from);
      const int64_t n = sums.workers + std::min(zeros - from, kMaxZeros);
      if (n > 0) hipLaunchKernelGGL(few, dim3(unsigned(n)), dim3(kSumNT), 0, s, sums, a.ids, int(a.T), blocks, a.err_flag);
      sums.workers = 0;
    }
    return;
  }
  const int owners = embed_owners(a.V), log_owners = __builtin_ctz(unsigned(owners));
  hipLaunchKernelGGL(k_embed_sort, dim3(unsigned(owners)), dim3(kSortNT), 0, s, a.ids, a.T, a.V, log_owners, w.sorted, w.n, w.there, a.err_flag);
  const int64_t most = int64_t(kWorkers) * compute_units() * kSumWaves;   // waves
  while ((2 << sums.log_split) <= blocks && (a.T << (sums.log_split + 1)) <= most) ++sums.log_split;
  sums.workers = int(std::min(most, std::max<int64_t>(a.T << sums.log_split, 1)) + kSumWaves - 1) / kSumWaves;
  const auto sum = vec ? k_embed_sum<DT, OUT, true> : k_embed_sum<DT, OUT, false>;
  hipLaunchKernelGGL(sum, dim3(unsigned(sums.workers + std::min(zeros, kMaxZeros))), dim3(kSumNT), 0, s, sums);
  sums.workers = 0;
  for (int64_t from = kMaxZeros; from < zeros; from += kMaxZeros) {
    sums.zeros_from = uint64_t(from);
    hipLaunchKernelGGL(sum, dim3(unsigned(std::min(zeros - from, kMaxZeros))), dim3(kSumNT), 0, s, sums);
  }
  hipLaunchKernelGGL(k_embed_join<OUT>, dim3(unsigned(kWorkers * compute_units())), dim3(kSumNT), 0, s, sums);
}

template <int DT>
static void embed_fwd_launch(const void* table, int V, int H, const int32_t* ids, int64_t T, float scale, void* out, int64_t ld_out,
                             int32_t* err_flag, hipStream_t s) {
  const bool vec = H >= Storage<DT>::kPerVec;
  const int per = vec ? (H + Storage<DT>::kPerVec - 1) / Storage<DT>::kPerVec : H, rows = std::max(kLookNT / per, 1);
  const auto fwd = rows == 1 ? k_embed_fwd<DT, true, false> : vec ? k_embed_fwd<DT, true, true> : k_embed_fwd<DT, false, true>;
  hipLaunchKernelGGL(fwd, dim3(unsigned((T + rows - 1) / rows)), dim3(kLookNT), 0, s, table, V, H, ids, T, rows, scale, out, ld_out, err_flag);
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
