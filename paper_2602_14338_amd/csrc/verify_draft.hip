// Verification of drafted tokens against the policy's rows, from given random numbers.
//
// Two launches.  The first forms the running sums of every row that can matter, (target rows up to the count of drafted
// tokens, the draft rows in front), a row split over several workgroups when there are few.  The second finds, in every
// workgroup of a sequence alike, the first position whose uniform number is not below p / q, and its slice of the vocabulary for the
// largest max(0, p - q) / noise there; the slices meet in one 64-bit maximum of (score, lowest id), which does not
// depend on their order, and the workgroup that comes last writes the sequence's outputs.
#include <algorithm>

#include "row_scan.h"

namespace aero {

constexpr int kVerifyParts = 8;   // most parts of a row in the first launch

struct VerifyArgs {
  const void *target, *draft;
  int B, G, V;
  int64_t ld;
  const int32_t *tokens, *count;
  const float *uniform, *noise;
  int32_t* accepted;
  int32_t* out;
  float* logprob;
  int32_t* err_flag;
  SoftSum* sums;                    // [B * (2 G + 1)][parts]: target rows, then draft rows
  unsigned long long* best;         // [B][2]: of the residual, of p itself
  int32_t* arrived;                 // [B]
  int parts;
};

// Drafted tokens of a sequence that count: up to its count, and to the first id outside the vocabulary.  -1: idle.  Every lane of the
// wave gets it; token = this lane's drafted id (lanes in front of the result).
__device__ __forceinline__ int drafted(const VerifyArgs& a, int b, int lane, int& token, int32_t& flags) {
  const int n = a.count ? a.count[b] : a.G;
  flags = 0;
  token = -1;
  if (n < 0 || n > a.G) {
    if (n > a.G) flags = AERO_DERR_BAD_COUNT;
    return -1;
  }
  if (lane < n) token = a.tokens[int64_t(b) * a.G + lane];
  const uint64_t bad = __builtin_amdgcn_ballot_w64(lane < n && (token < 0 || token >= a.V));
  if (!bad) return n;
  const int first = __builtin_ctzll(bad);
  if (__builtin_amdgcn_readlane(token, first) >= a.V) flags = AERO_DERR_BAD_TARGET;
  return first;
}

template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_verify_rows(VerifyArgs a) {
  constexpr int E = RowView<DT, VEC>::E, kAhead = VEC ? 4 : 8;
  __shared__ SoftSum s_sum[NT / kWave];
  const int tid = threadIdx.x, part = blockIdx.y, parts = gridDim.y;
  const int64_t r = blockIdx.x, n_target = int64_t(a.B) * (a.G + 1);
  const bool is_target = r < n_target;
  const int width = is_target ? a.G + 1 : a.G;
  const int64_t rr = is_target ? r : r - n_target;
  const int b = int(rr / width), i = int(rr % width);
  if (is_target && i == 0 && part == 0 && tid == 0) {
    a.best[2 * b] = 0;
    a.best[2 * b + 1] = 0;
    a.arrived[b] = 0;
  }
  int token;
  int32_t flags;
  const int n = drafted(a, b, tid % kWave, token, flags);
  if (is_target ? i > n : i >= n) return;   // uniform
  const RowView<DT, VEC> row(is_target ? a.target : a.draft, rr, a.ld, a.V);
  const int per = (row.nvec + parts - 1) / parts;
  const int first = min(part * per, row.nvec), last = min(first + per, row.nvec);
  const int jr = part == 0 ? row.ragged() : -1;
  SoftSum st = soft_identity();
  if (jr >= 0) {
    float z[1] = {row.at(jr)};
    soft_update<1>(st, z);
  }
  int k = first + tid;
  for (; k + (kAhead - 1) * NT < last; k += kAhead * NT) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = row.load(k + u * NT);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float z[E];
      row.unpack(v[u], z);
      soft_update<E>(st, z);
    }
  }
  for (; k < last; k += NT) {
    float z[E];
    row.unpack(row.load(k), z);
    soft_update<E>(st, z);
  }
  st = soft_block_reduce<NT>(st, s_sum);
  if (tid == 0) a.sums[r * parts + part] = st;
}

__device__ __forceinline__ SoftSum row_sum(const VerifyArgs& a, int64_t r) {
  SoftSum st = soft_identity();
  for (int p = 0; p < a.parts; ++p) st = soft_merge(st, a.sums[r * a.parts + p]);
  return st;
}

// Largest score so far and its column.
struct Drawn {
  float score;
  int j;
};
__device__ __forceinline__ void race(Drawn& d, float score, int j) {
  if (score > d.score) d = Drawn{score, j};   // columns ascend within a thread
}
__device__ __forceinline__ uint64_t drawn_key(Drawn d) {
  return d.score > 0.f ? (uint64_t(__float_as_uint(d.score)) << 32) | uint32_t(~d.j) : 0;
}
// E elements from column j on, or floats, at any element's alignment.
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(1)));
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
template <int DT, bool VEC> __device__ __forceinline__ u32x4_t load_elts(const char* row, int j) {
  if constexpr (VEC) return *reinterpret_cast<const u32x4_any_t*>(row + int64_t(j) * Storage<DT>::kBytes);
  else return u32x4_t{__float_as_uint(load_elt<DT>(row, j)), 0u, 0u, 0u};
}
template <int E> __device__ __forceinline__ void load_floats(const float* x, float (&y)[E]) {
  if constexpr (E == 1) {
    y[0] = x[0];
  } else {
#pragma unroll
    for (int k = 0; k < E; k += 4) {
      const f32x4_any_t v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any_t*>(x + k));
      y[k] = v.x; y[k + 1] = v.y; y[k + 2] = v.z; y[k + 3] = v.w;
    }
  }
}
template <int NT> __device__ __forceinline__ uint64_t block_max_u64(uint64_t x, uint64_t* lds) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const uint64_t y = __shfl_xor(x, m, kWave);
    x = y > x ? y : x;
  }
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = x;
  __syncthreads();
  x = lds[0];
#pragma unroll
  for (int w = 1; w < NT / kWave; ++w) x = lds[w] > x ? lds[w] : x;
  return x;
}

template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_verify_draw(VerifyArgs a) {
  constexpr int E = RowView<DT, VEC>::E;
  __shared__ uint64_t s_key[2][NT / kWave];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid % kWave, b = blockIdx.x, part = blockIdx.y, parts = gridDim.y;
  int token;
  int32_t flags;
  const int count = drafted(a, b, lane, token, flags);
  if (part == 0 && tid == 0 && flags && a.err_flag) atomicOr(a.err_flag, flags);
  int32_t* const out = a.out + int64_t(b) * (a.G + 1);
  float* const lp_out = a.logprob ? a.logprob + int64_t(b) * (a.G + 1) : nullptr;
  if (count < 0) {
    if (part == 0) {
      if (tid == 0) a.accepted[b] = 0;
      for (int i = tid; i <= a.G; i += NT) {
        out[i] = -1;
        if (lp_out) lp_out[i] = 0.f;
      }
    }
    return;
  }
  // ---- lane i: position i ----
  const int64_t n_target = int64_t(a.B) * (a.G + 1);
  bool ok = false;
  double lp = 0.0;
  if (lane < count) {
    const int64_t rt = int64_t(b) * (a.G + 1) + lane, rd = int64_t(b) * a.G + lane;
    lp = double(load_elt<DT>(row_ptr<DT>(a.target, rt, a.ld), token)) - soft_lse(row_sum(a, rt));
    double q = 1.0;
    if (a.draft) q = exp(double(load_elt<DT>(row_ptr<DT>(a.draft, rd, a.ld), token)) - soft_lse(row_sum(a, n_target + rd)));
    ok = double(a.uniform[rd]) * q < exp(lp);
  }
  const int n = __builtin_ctzll(~__builtin_amdgcn_ballot_w64(ok));   // at most 63 positions
  const bool refused = n < count;
  const int own = refused && !a.draft ? __builtin_amdgcn_readlane(token, n) : -1;   // the whole of q

  // ---- the draw: this workgroup's slice of row n ----
  const int64_t rt = int64_t(b) * (a.G + 1) + n, rd = int64_t(b) * a.G + n;
  const SoftSum pt = row_sum(a, rt);
  const double lse = soft_lse(pt);
  Drawn left{0.f, 0}, whole{0.f, 0};
  if (lse - lse == 0.0) {   // finite
    SoftSum qt = soft_identity();
    if (refused && a.draft) qt = row_sum(a, n_target + rd);
    const double lse_q = soft_lse(qt);
    const bool minus = lse_q - lse_q == 0.0;
    const float op = -pt.o, sp = 1.f / pt.s, oq = minus ? -qt.o : 0.f, sq = minus ? 1.f / qt.s : 0.f;
    const RowView<DT, VEC> prow(a.target, rt, a.ld, a.V);
    const char* const qrow = minus ? row_ptr<DT>(a.draft, rd, a.ld) : nullptr;
    const float* const noise = a.noise + int64_t(b) * a.V;
    auto consider = [&](float z, float y, float e, int j) {
#pragma clang fp contract(off)   // equal probabilities leave nothing
      const float p = sp * exp2_fast(fmaf(z, kLog2e, op)), chance = __builtin_amdgcn_rcpf(e);
      const float q = sq * exp2_fast(fmaf(y, kLog2e, oq)), r = j == own ? 0.f : p - q;
      race(left, r * chance, j);
      race(whole, p * chance, j);
    };
    const int per = (prow.nvec + parts - 1) / parts;
    const int first = min(part * per, prow.nvec), last = min(first + per, prow.nvec);
    for (int i = first + tid; i < last; i += NT) {
      const int j = prow.column(i);
      float z[E], y[E], e[E];
      const u32x4_t zv = prow.load_again(i);
      u32x4_t yv = {0u, 0u, 0u, 0u};
      if (minus) yv = load_elts<DT, VEC>(qrow, j);
      load_floats<E>(noise + j, e);
      prow.unpack(zv, z);
      prow.unpack(yv, y);
#pragma unroll
      for (int k = 0; k < E; ++k) consider(z[k], y[k], e[k], j + k);
    }
    const int jr = part == 0 ? prow.ragged() : -1;
    if (jr >= 0) {   // a tie goes to the lower id, which is not the later one here
      Drawn l = left, w = whole;
      left = whole = Drawn{0.f, 0};
      consider(prow.at(jr), minus ? load_elt<DT>(qrow, jr) : 0.f, noise[jr], jr);
      left = drawn_key(l) > drawn_key(left) ? l : left;
      whole = drawn_key(w) > drawn_key(whole) ? w : whole;
    }
  }
  const uint64_t k_left = block_max_u64<NT>(drawn_key(left), s_key[0]);
  const uint64_t k_whole = block_max_u64<NT>(drawn_key(whole), s_key[1]);
  if (tid == 0) {
    if (k_left) atomicMax(&a.best[2 * b], (unsigned long long)k_left);
    if (k_whole) atomicMax(&a.best[2 * b + 1], (unsigned long long)k_whole);
    __threadfence();
    s_last = atomicAdd(&a.arrived[b], 1) == parts - 1;
  }
  __syncthreads();
  if (!s_last || tid >= kWave) return;
  __threadfence();
  uint64_t key = atomicMax(&a.best[2 * b], 0ull);
  if (!key && refused) key = atomicMax(&a.best[2 * b + 1], 0ull);
  const int drawn = key ? int(~uint32_t(key)) : -1;
  const float drawn_lp = drawn >= 0 ? float(double(load_elt<DT>(row_ptr<DT>(a.target, rt, a.ld), drawn)) - lse) : 0.f;
  if (lane == 0) a.accepted[b] = n;
  if (lane <= a.G) {
    out[lane] = lane < n ? token : lane == n ? drawn : -1;
    if (lp_out) lp_out[lane] = lane < n ? float(lp) : lane == n ? drawn_lp : 0.f;
  }
}

static size_t verify_sum_bytes(int64_t rows) { return (size_t(2 * rows) * kVerifyParts * sizeof(SoftSum) + 255) / 256 * 256; }
size_t verify_workspace_bytes(int64_t rows, int32_t V, int32_t B) {
  (void)V;
  return verify_sum_bytes(rows) + (size_t(B > 0 ? B : 0) * 20 + 255) / 256 * 256 + 256;
}

template <int DT, bool VEC> static void verify_launch(VerifyArgs a, hipStream_t s) {
  constexpr int NT = 512;
  const int64_t rows = int64_t(a.B) * (a.G + 1) + (a.draft ? int64_t(a.B) * a.G : 0);
  const int nvec = a.V / RowView<DT, VEC>::E;
  a.parts = int(std::max<int64_t>(1, std::min<int64_t>({kVerifyParts, 2 * compute_units() / rows, nvec / (4 * NT)})));
  hipLaunchKernelGGL((k_verify_rows<NT, DT, VEC>), dim3(unsigned(rows), unsigned(a.parts)), dim3(NT), 0, s, a);
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(4 * compute_units() / a.B, nvec / NT)));
  hipLaunchKernelGGL((k_verify_draw<NT, DT, VEC>), dim3(unsigned(a.B), unsigned(parts)), dim3(NT), 0, s, a);
}

}  // namespace aero

extern "C" aero_status aero_verify_draft(const void* target_logits, const void* draft_logits, int32_t dtype, int32_t B, int32_t G,
                                         int32_t V, int64_t ld, const int32_t* draft_tokens, const int32_t* draft_count,
                                         const float* uniform, const float* noise, int32_t* accepted, int32_t* tokens, float* logprob,
                                         int32_t* err_flag, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace aero;
  if (B < 0 || G < 0 || V < 1 || V > (1 << 24) || ld < V) return AERO_ERR_SHAPE;
  if (G > AERO_DRAFT_MAX) return AERO_ERR_LIMIT;
  if (!grid_fits(int64_t(B) * (2 * G + 1), 1024)) return AERO_ERR_SHAPE;
  if (!storage_dtype_ok(dtype)) return AERO_ERR_DTYPE;
  if (B == 0) return AERO_OK;
  if (!target_logits || !noise || !accepted || !tokens || (G > 0 && (!draft_tokens || !uniform))) return AERO_ERR_NULL;
  const int64_t rows = int64_t(B) * (G + 1);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < verify_workspace_bytes(rows, V, B))
    return AERO_ERR_WORKSPACE;
  char* const ws = reinterpret_cast<char*>(workspace);
  unsigned long long* const best = reinterpret_cast<unsigned long long*>(ws + verify_sum_bytes(rows));
  const VerifyArgs a{target_logits, G > 0 ? draft_logits : nullptr, B, G, V, ld, draft_tokens, draft_count, uniform, noise, accepted, tokens,
                     logprob, err_flag, reinterpret_cast<SoftSum*>(ws), best, reinterpret_cast<int32_t*>(best + 2 * size_t(B)), 1};
  const bool vec = rows_alike(target_logits, nullptr, storage_bytes(dtype)) && rows_alike(a.draft, nullptr, storage_bytes(dtype));
  const hipStream_t s = as_stream(stream);
  switch (dtype) {
    case AERO_BF16: vec ? verify_launch<kBF16, true>(a, s) : verify_launch<kBF16, false>(a, s); break;
    case AERO_F16: vec ? verify_launch<kF16, true>(a, s) : verify_launch<kF16, false>(a, s); break;
    case AERO_F8E4M3: vec ? verify_launch<kF8, true>(a, s) : verify_launch<kF8, false>(a, s); break;
    default: vec ? verify_launch<kF32, true>(a, s) : verify_launch<kF32, false>(a, s);
  }
  return launch_status();
}
