// Embedding rows looked up and scaled, and the gradient of the table from tokens sorted by id.
//
// The sort is a launch of independent workgroups, each of which owns the ids that are alike modulo their number and goes
// over all tokens twice: once to count (its own ids one by one, what lies in front of them as a whole), once to place its
// tokens, in ascending order within an id.  Every token is read by every workgroup, out of the caches; nothing passes
// between workgroups and there are no counters whose order could show.  What a frequent id has to add up is cut into
// pieces of kPiece tokens, summed in a second launch and, where there is more than one, joined in order in a third.  Rows
// that no token has are zeroed in the second launch, beside the sums, so that the sort has nothing to wait for.
#include <algorithm>

#include "aero_device.h"

namespace aero {

// One workgroup per token row.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void k_embed_fwd(const void* __restrict__ table, int V, int H, const int32_t* __restrict__ ids,
                                                   float scale, void* __restrict__ out, int64_t ld_out,
                                                   int32_t* __restrict__ err_flag) {
  constexpr int E = VEC ? Storage<DT>::kPerVec : 1;
  const int64_t t = blockIdx.x;
  const int id = ids[t];
  if (id >= V && threadIdx.x == 0 && err_flag) atomicOr(err_flag, AERO_DERR_BAD_TARGET);
  const bool there = id >= 0 && id < V;
  const char* const src = row_ptr<DT>(table, there ? id : 0, H);
  char* const dst = row_ptr<DT>(out, t, ld_out);
  for (int i = threadIdx.x; i < H / E; i += 256) {
    if constexpr (VEC) {
      u32x4_t v = {0u, 0u, 0u, 0u};
      if (there) {
        float x[E];
        unpack_vec<DT>(reinterpret_cast<const u32x4_t*>(src)[i], x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] *= scale;
        v = pack_vec<DT>(x);
      }
      reinterpret_cast<u32x4_t*>(dst)[i] = v;
    } else {
      store_elt<DT>(dst, i, there ? scale * load_elt<DT>(src, i) : 0.f);
    }
  }
}

// ---- gradient ----
constexpr int kSortNT = 1024, kSortAhead = 4, kSortChunk = kSortNT * kSortAhead;
constexpr int kLogBins = 10, kBins = 1 << kLogBins;   // ids of a sorting workgroup
constexpr int kMinOwners = 256;  // sorting workgroups, a power of two
constexpr int kPiece = 32;       // tokens that one wave adds up
constexpr int kFillParts = 4;    // workgroups that zero the rows of an owner

// A run of sorted tokens: pieces of an id.  Slot s describes the piece whose first piece's tokens start at sorted position
// s - piece; slots that no piece has are empty (count 0).
struct Piece {
  int32_t id, start, count;
  int32_t part;   // 0: the id has one piece; else 1 + the piece's number
  int32_t whole;  // tokens of the id
  int32_t row;    // where the piece's sum goes when there are several
  int32_t pad[2];
};

static int embed_owners(int32_t V) {
  int owners = kMinOwners;
  while (int64_t(owners) * kBins < V) owners *= 2;
  return owners;
}
struct EmbedWorkspace {
  int32_t* order;   // [T] tokens sorted by id
  Piece* piece;     // [T]
  int32_t* n_empty; // [owners]
  int32_t* empty;   // [owners][kBins] ids that no token has
  float* partial;   // [2 (T / kPiece + 1)][H]
  size_t bytes;
};
static EmbedWorkspace embed_workspace(void* base, int64_t T, int32_t V, int64_t H) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  char* p = reinterpret_cast<char*>(base);
  EmbedWorkspace w;
  w.order = reinterpret_cast<int32_t*>(p);
  size_t at = up(size_t(T) * 4);
  w.piece = reinterpret_cast<Piece*>(p + at);
  at += up(size_t(T) * sizeof(Piece));
  const size_t owners = embed_owners(V);
  w.n_empty = reinterpret_cast<int32_t*>(p + at);
  at += up(owners * 4);
  w.empty = reinterpret_cast<int32_t*>(p + at);
  at += up(owners * kBins * 4);
  w.partial = reinterpret_cast<float*>(p + at);
  at += up(size_t(2 * (T / kPiece + 1)) * size_t(H) * 4);
  w.bytes = at + 256;
  return w;
}
size_t embedding_workspace_bytes(int64_t T, int32_t V, int32_t H) {
  return embed_workspace(nullptr, T, V > 0 ? V : 1, H > 0 ? H : 0).bytes;
}

// Workgroup g owns the ids with id % owners == g.  Its ids without a token go to empty[g * kBins ...], their number to n_empty[g].
__global__ __launch_bounds__(kSortNT) void k_embed_sort(const int32_t* __restrict__ ids, int64_t T, int V, int log_owners,
                                                        int32_t* __restrict__ order, Piece* __restrict__ pieces,
                                                        int32_t* __restrict__ empty, int32_t* __restrict__ n_empty,
                                                        int32_t* __restrict__ err_flag) {
  __shared__ int s_count[kBins], s_at[kBins];
  __shared__ int s_wave[kSortNT / kWave];
  __shared__ int s_none;
  __shared__ int32_t s_tok[kSortChunk];
  __shared__ __align__(16) uint16_t s_bin[kSortChunk];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = blockIdx.x, mask = (1 << log_owners) - 1;
  const int bins = (V - g + mask) >> log_owners;   // ids g, g + owners, ... below V
  s_count[tid] = 0;
  if (tid == 0) s_none = 0;
  __syncthreads();
  // ---- count ----
  int before = 0;
  bool bad = false;
  for (int64_t t0 = 0; t0 < T; t0 += 2 * kSortChunk) {
    int id[2 * kSortAhead];
#pragma unroll
    for (int u = 0; u < 2 * kSortAhead; ++u) {
      const int64_t t = t0 + u * kSortNT + tid;
      id[u] = t < T ? ids[t] : -1;
    }
#pragma unroll
    for (int u = 0; u < 2 * kSortAhead; ++u) {
      bad |= id[u] >= V;
      const bool in = id[u] >= 0 && id[u] < V;
      const int owner = id[u] & mask;
      before += in && owner < g;
      if (in && owner == g) atomicAdd(&s_count[id[u] >> log_owners], 1);
    }
  }
  if (g == 0 && bad && err_flag) atomicOr(err_flag, AERO_DERR_BAD_TARGET);
  before = wave_sum_i(before);
  if (lane == 0) s_wave[wave] = before;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < kSortNT / kWave; ++w) base += s_wave[w];
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
  if (lane == kWave - 1) s_wave[wave] = incl;
  __syncthreads();
  int start = base + incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kSortNT / kWave; ++w) {
    if (w < wave) start += s_wave[w];
    total += s_wave[w];
  }
  s_at[tid] = start;
  // ---- pieces ----
  // (behind the last owner's tokens lie the slots of tokens that no id counts)
  const int64_t slots = g == int(gridDim.x) - 1 ? T - base : total;
  for (int64_t k = tid; k < slots; k += kSortNT) pieces[base + k].count = 0;
  __syncthreads();
  const int id_mine = (tid << log_owners) + g;
  if (mine > 0) {
    const int np = (mine + kPiece - 1) / kPiece;
    for (int k = 0; k < np; ++k)
      pieces[start + k] = Piece{id_mine, start + k * kPiece, min(kPiece, mine - k * kPiece), np == 1 ? 0 : 1 + k, mine,
                                2 * (start / kPiece) + k, {0, 0}};
  } else if (tid < bins) {
    empty[g * kBins + atomicAdd(&s_none, 1)] = id_mine;   // rows of zeros: their order is nothing's
  }
  // ---- place, in order ----
  for (int64_t t0 = 0; total > 0 && t0 < T; t0 += kSortChunk) {
    // a thread's tokens follow each other, so that (thread, u) is their order
    int id[kSortAhead];
    bool own[kSortAhead];
    int ahead = 0, in_wave = 0;
#pragma unroll
    for (int u = 0; u < kSortAhead; ++u) {
      const int64_t t = t0 + tid * kSortAhead + u;
      id[u] = t < T ? ids[t] : -1;
      own[u] = id[u] >= 0 && id[u] < V && (id[u] & mask) == g;
      const uint64_t m = __builtin_amdgcn_ballot_w64(own[u]);
      ahead += __popcll(m & ((uint64_t(1) << lane) - 1));
      in_wave += __popcll(m);
    }
    if (lane == 0) s_wave[wave] = in_wave;
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int w = 0; w < kSortNT / kWave; ++w) {
      if (w < wave) ahead += s_wave[w];
      n += s_wave[w];
    }
#pragma unroll
    for (int u = 0; u < kSortAhead; ++u) {
      if (own[u]) {
        s_tok[ahead] = int32_t(t0 + tid * kSortAhead + u);
        s_bin[ahead] = uint16_t(id[u] >> log_owners);
        ++ahead;
      }
    }
    __syncthreads();
    // 64 at a time by the first wave: a token's place is its id's next one plus the lanes in front with the same id
    if (wave == 0) {
      for (int k0 = 0; k0 < n; k0 += kWave) {
        const int k = k0 + lane;
        const bool in = k < n;
        const int bin = in ? s_bin[k] : 0;
        uint64_t same = __builtin_amdgcn_ballot_w64(in);
#pragma unroll
        for (int bit = 0; bit < kLogBins; ++bit) {
          const uint64_t m = __builtin_amdgcn_ballot_w64((bin >> bit & 1) != 0);
          same &= (bin >> bit & 1) != 0 ? m : ~m;
        }
        if (in) {
          const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
          const int at = s_at[bin];
          order[at + rank] = s_tok[k];
          if (rank == 0) s_at[bin] = at + __popcll(same);   // read above by every lane of the id: one wave, in step
        }
      }
    }
    __syncthreads();
  }
  if (tid == 0) n_empty[g] = s_none;
}

// N sums, scaled, to consecutive columns of the table: added to what is there, or in its place.
template <int OUT, int N> __device__ __forceinline__ void put_sums(char* at, const float (&sum)[N], float scale, bool accumulate) {
  constexpr int kBytes = N * Storage<OUT>::kBytes;
  float x[N];
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = scale * sum[e];
  if constexpr (kBytes % 16 == 0) {
    constexpr int E = Storage<OUT>::kPerVec;
#pragma unroll
    for (int v = 0; v < kBytes / 16; ++v) {
      u32x4_t* const p = reinterpret_cast<u32x4_t*>(at) + v;
      float y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = 0.f;
      if (accumulate) unpack_vec<OUT>(*p, y);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = accumulate ? y[e] + x[v * E + e] : x[v * E + e];
      __builtin_nontemporal_store(pack_vec<OUT>(y), p);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) store_elt<OUT>(at, e, accumulate ? load_elt<OUT>(at, e) + x[e] : x[e]);
  }
}

constexpr int kSumNT = 256, kSumWaves = kSumNT / kWave, kRowsAhead = 4;
// The first n_sum workgroups: wave (slot, column block), the sum of a piece's rows, to the table or, of an id with several pieces, to
// `partial`.  The others (not with accumulate): rows of zeros for the ids that no token has.  VEC: dout in 16-byte vectors, and the table
// where a lane's sums are whole vectors of it.
template <int DT, int OUT, bool VEC>
__global__ __launch_bounds__(kSumNT) void k_embed_sum(const void* __restrict__ dout, int64_t ld, int H, int64_t T, int n_sum, int n_owners,
                                                      const int32_t* __restrict__ order, const Piece* __restrict__ pieces,
                                                      const int32_t* __restrict__ empty, const int32_t* __restrict__ n_empty, float scale,
                                                      int accumulate, float* __restrict__ partial, void* __restrict__ table) {
  constexpr int E = VEC ? Storage<DT>::kPerVec : 1;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  if (int(blockIdx.x) >= n_sum) {
    const int part = (int(blockIdx.x) - n_sum) * gridDim.y + blockIdx.y, g = part / kFillParts;
    if (g >= n_owners) return;
    const int n = n_empty[g];
    for (int k = part % kFillParts * kSumWaves + wave; k < n; k += kFillParts * kSumWaves) {
      const int64_t id = empty[g * kBins + k];
      char* const row = row_ptr<OUT>(table, id, H);
      const RowGeom geom = row_geom<OUT>(table, id, H, H);
      const u32x4_t zero = {0u, 0u, 0u, 0u};
      for (int i = lane; i < geom.nvec; i += kWave)
        __builtin_nontemporal_store(zero, reinterpret_cast<u32x4_t*>(row + geom.head * Storage<OUT>::kBytes) + i);
      const int j = ragged_elt<OUT>(geom, H, lane);
      if (j >= 0) store_elt<OUT>(row, j, 0.f);
    }
    return;
  }
  const int64_t slot = int64_t(blockIdx.x) * kSumWaves + wave;
  if (slot >= T) return;
  const int count = pieces[slot].count;
  if (count == 0) return;
  const Piece p = pieces[slot];
  const int own = lane < kPiece && lane < count ? order[p.start + lane] : 0;   // lane k: the piece's k-th token
  for (int c = (blockIdx.y * kWave + lane) * E; c < H; c += gridDim.y * kWave * E) {
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.f;
    for (int k0 = 0; k0 < count; k0 += kRowsAhead) {
      float x[kRowsAhead][E];
      u32x4_t v[kRowsAhead];
#pragma unroll
      for (int k = 0; k < kRowsAhead; ++k) {
        const char* const row = row_ptr<DT>(dout, __builtin_amdgcn_readlane(own, min(k0 + k, count - 1)), ld, c);
        if constexpr (VEC) v[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row));
        else x[k][0] = load_elt<DT>(row, 0);
      }
#pragma unroll
      for (int k = 0; k < kRowsAhead; ++k) {
        if constexpr (VEC) unpack_vec<DT>(v[k], x[k]);
        if (k0 + k < count) {   // uniform
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] += x[k][e];
        }
      }
    }
    if (p.part == 0) {
      put_sums<OUT, E>(row_ptr<OUT>(table, p.id, H, c), sum, scale, accumulate != 0);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) partial[size_t(p.row) * H + c + e] = sum[e];
    }
  }
}

// Workgroup (unit, column block): the id with several pieces whose tokens start in the unit's kPiece sorted positions (at most one
// does: it has more tokens than the unit has positions).
template <int OUT>
__global__ __launch_bounds__(kSumNT) void k_embed_join(int64_t T, int H, const Piece* __restrict__ pieces, float scale, int accumulate,
                                                       const float* __restrict__ partial, void* __restrict__ table) {
  static_assert(kPiece <= kWave, "a lane per position");
  const int lane = threadIdx.x % kWave;
  const int64_t slot = int64_t(blockIdx.x) * kPiece + lane;
  const bool head = lane < kPiece && slot < T && pieces[slot].count > 0 && pieces[slot].part == 1;
  const uint64_t first = __builtin_amdgcn_ballot_w64(head);
  if (!first) return;
  const Piece p = pieces[int64_t(blockIdx.x) * kPiece + __builtin_ctzll(first)];
  const int np = (p.whole + kPiece - 1) / kPiece;
  for (int c = blockIdx.y * kSumNT + threadIdx.x; c < H; c += gridDim.y * kSumNT) {
    float sum[1] = {0.f};
    int k = 0;
    for (; k + 8 <= np; k += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = partial[size_t(p.row + k + u) * H + c];
#pragma unroll
      for (int u = 0; u < 8; ++u) sum[0] += x[u];
    }
    for (; k < np; ++k) sum[0] += partial[size_t(p.row + k) * H + c];
    put_sums<OUT, 1>(row_ptr<OUT>(table, p.id, H, c), sum, scale, accumulate != 0);
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

template <int DT, int OUT> static void embed_bwd_launch(const EmbedArgs& a, void* workspace, hipStream_t s) {
  const EmbedWorkspace w = embed_workspace(workspace, a.T, a.V, a.H);
  const int owners = embed_owners(a.V), log_owners = __builtin_ctz(unsigned(owners));
  hipLaunchKernelGGL(k_embed_sort, dim3(unsigned(owners)), dim3(kSortNT), 0, s, a.ids, a.T, a.V, log_owners, w.order, w.piece, w.empty,
                     w.n_empty, a.err_flag);
  constexpr int E = Storage<DT>::kPerVec;
  const bool vec = a.H % E == 0 && a.ld % E == 0 && reinterpret_cast<uintptr_t>(a.dout) % 16 == 0 &&
                   a.H % Storage<OUT>::kPerVec == 0 && reinterpret_cast<uintptr_t>(a.table) % 16 == 0;
  const int per_wave = kWave * (vec ? E : 1);
  const int columns = std::min(8, (a.H + per_wave - 1) / per_wave), n_sum = int((a.T + kSumWaves - 1) / kSumWaves);
  const int fill = a.accumulate ? 0 : (owners * kFillParts + columns - 1) / columns;
  const auto sum = vec ? k_embed_sum<DT, OUT, true> : k_embed_sum<DT, OUT, false>;
  if (n_sum + fill > 0)
    hipLaunchKernelGGL(sum, dim3(unsigned(n_sum + fill), unsigned(columns)), dim3(kSumNT), 0, s, a.dout, a.ld, a.H, a.T, n_sum, owners, w.order,
                       w.piece, w.empty, w.n_empty, a.scale, a.accumulate, w.partial, a.table);
  if (a.T > kPiece)
    hipLaunchKernelGGL(k_embed_join<OUT>, dim3(unsigned((a.T + kPiece - 1) / kPiece), unsigned(std::min(8, (a.H + kSumNT - 1) / kSumNT))),
                       dim3(kSumNT), 0, s, a.T, a.H, w.piece, a.scale, a.accumulate, w.partial, a.table);
}

template <int DT>
static void embed_fwd_launch(const void* table, int V, int H, const int32_t* ids, int64_t T, float scale, void* out, int64_t ld_out,
                             int32_t* err_flag, hipStream_t s) {
  constexpr int E = Storage<DT>::kPerVec;
  const bool vec = H % E == 0 && ld_out % E == 0 && reinterpret_cast<uintptr_t>(table) % 16 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
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
