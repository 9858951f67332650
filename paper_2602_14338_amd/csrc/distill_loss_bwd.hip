// Distillation from a teacher's top logits: divergence of each row from its list, and the gradient row.
//
// With q = softmax(z), the list's ids i_k with probabilities p_k and everything else as one event of probability p_r:
//   L = sum_k p_k (ln p_k - ln q(i_k)) + p_r (ln p_r - ln q_r),   P = sum p + p_r,
//   dL/dz_j = P q_j - p_j (listed),  (P - p_r / q_r) q_j (others);
// the renormalised form is p_k / sum p with p_r = 0.  So a gradient row is one multiple of the exponentials, replaced at
// the K listed places.
//
// q_r is what a converging drafter makes small, and 1 - sum q(i_k) would leave nothing of it: the sum over the row leaves the
// listed places out (they count as masked while it runs) and their K exponentials are added to it.  Each thread knows from a
// chain of the entries that fall into its vectors which of them hold listed places, so that all other vectors pay one
// comparison.
#include "row_scan.h"

namespace aero {

constexpr int kListMax = AERO_TOPK_MAX;
constexpr int kNowhere = 0x7fffffff;

// The entries of a row's list by the thread that looks after their place.
template <int NT> struct ListPlaces {
  int32_t head[NT];          // first entry of a thread's chain, -1: none
  int32_t next[kListMax];
  int32_t vec[kListMax];     // vector of the place; nvec: the ragged element of its thread
  uint8_t elt[kListMax];
  float p[kListMax];         // w grad_scale p_k once the row's terms are known
  int bad;
};

// Next vector of this thread from `after` on (exclusive) that holds a listed place.
template <int NT> __device__ __forceinline__ int next_listed(const ListPlaces<NT>& l, int after) {
  int v = kNowhere;
  for (int k = l.head[threadIdx.x]; k >= 0; k = l.next[k]) {
    const int at = l.vec[k];
    if (at > after && at < v) v = at;
  }
  return v;
}

template <int NT> __device__ __forceinline__ double block_sum_d(double x, double* lds /*[NT/64]*/) {
  x = wave_sum_d(x);
  constexpr int kWaves = NT / kWave;
  if constexpr (kWaves > 1) {
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += lds[w];
    __syncthreads();
  }
  return x;
}

struct DistillArgs {
  const void* logits;
  int64_t T;
  int V;
  int64_t ld;
  const int32_t* index;
  const float* logprob;
  int K;
  const float* weight;
  int tail;
  float grad_scale;
  float *term, *row_loss;
  void* dlogits;
  int32_t* err_flag;
};

// One workgroup per row, which is read twice.  VEC: 16-byte vectors (logits and dlogits at the same offset from 16 bytes).
template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(NT) void k_distill_row(DistillArgs a) {
  using View = RowView<DT, VEC>;
  constexpr int E = View::E, kAhead = 4, kWaves = NT / kWave;
  __shared__ ListPlaces<NT> list;
  __shared__ SoftSum s_sum[kWaves];
  __shared__ double s_dbl[kWaves];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, K = a.K;
  const float w = a.weight[t];
  const View row(a.logits, t, a.ld, a.V);
  const int nvec = row.nvec, jr = row.ragged();
  char* const drow = a.dlogits ? row_ptr<DT>(a.dlogits, t, a.ld) : nullptr;
  auto put = [&](int vec, const float (&d)[E]) {
    if constexpr (VEC)
      __builtin_nontemporal_store(pack_vec<DT>(d), reinterpret_cast<u32x4_t*>(drow + row.head * Storage<DT>::kBytes) + vec);
    else
      store_elt<DT>(drow, vec, d[0]);
  };
  auto finish = [&](float loss) {
    if (tid == 0) {
      a.term[t] = loss == 0.f ? 0.f : w * loss;   // an ignored row's weight may be anything
      if (a.row_loss) a.row_loss[t] = loss;
    }
  };
  auto zero_fill = [&]() {
    if (!drow) return;
    float zero[E];
#pragma unroll
    for (int e = 0; e < E; ++e) zero[e] = 0.f;
    for (int i = tid; i < nvec; i += NT) put(i, zero);
    if (jr >= 0) store_elt<DT>(drow, jr, 0.f);
  };
  if (w == 0.f) {   // uniform
    finish(0.f);
    zero_fill();
    return;
  }

  // ---- the list: probabilities, and whose vectors the places are in ----
  list.head[tid] = -1;
  if (tid == 0) list.bad = 0;
  __syncthreads();
  double mass = 0.0, own_p = 0.0, own_lp = 0.0;
  float own_z = -INFINITY;
  bool there = false;
  if (tid < K) {   // K <= NT
    const int j = a.index[t * K + tid];
    if (j >= a.V) list.bad = 1;
    there = j >= 0 && j < a.V;
    if (there) {
      own_lp = double(a.logprob[t * K + tid]);
      own_p = exp(own_lp);
      own_z = row.at(j);
      int vec = (j - row.head) / E, elt = (j - row.head) % E, owner = vec % NT;
      if constexpr (VEC) {
        if (j < row.head || vec >= nvec) {
          owner = j < row.head ? j : E + j - row.head - nvec * E;
          vec = nvec;
          elt = 0;
        }
      }
      list.vec[tid] = vec;
      list.elt[tid] = uint8_t(elt);
      list.next[tid] = atomicExch(&list.head[owner], tid);
    }
  }
  mass = block_sum_d<NT>(there ? own_p : 0.0, s_dbl);
  if (there)
    for (int k = list.next[tid]; k >= 0; k = list.next[k])
      if (list.vec[k] == list.vec[tid] && list.elt[k] == list.elt[tid]) list.bad = 1;
  const bool any = __syncthreads_or(there);
  if (list.bad && tid == 0 && a.err_flag) atomicOr(a.err_flag, AERO_DERR_BAD_TEACHER);
  if (list.bad || !any || (a.tail == AERO_TAIL_RENORM && mass == 0.0)) {   // uniform
    finish(0.f);
    zero_fill();
    return;
  }

  // ---- sum over the other places, then the list's part ----
  SoftSum st = soft_identity();
  {
    int listed = next_listed(list, -1);
    auto fold = [&](const u32x4_t& v, int i) {
      float z[E];
      View::unpack(v, z);
      if (__builtin_amdgcn_ballot_w64(i == listed) != 0 && i == listed) {
        for (int k = list.head[tid]; k >= 0; k = list.next[k])
          if (list.vec[k] == i) {
            const int own = list.elt[k];
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = e == own ? -INFINITY : z[e];
          }
        listed = next_listed(list, i);
      }
      soft_update<E>(st, z);
    };
    int i = tid;
    for (; i + (kAhead - 1) * NT < nvec; i += kAhead * NT) {
      u32x4_t v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = row.load(i + u * NT);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) fold(v[u], i + u * NT);
    }
    for (; i < nvec; i += NT) fold(row.load(i), i);
    if (jr >= 0 && listed != nvec) {
      float z[1] = {row.at(jr)};
      soft_update<1>(st, z);
    }
  }
  const SoftSum rest = soft_block_reduce<NT>(st, s_sum);
  __syncthreads();
  SoftSum own = soft_identity();
  if (there && !(own_z <= kMasked)) {
    float z[1] = {own_z};
    soft_update<1>(own, z);
  }
  own = soft_block_reduce<NT>(own, s_sum);
  const SoftSum all = soft_merge(rest, own);
  if (all.s == 0.f) {   // uniform: nothing but masked logits
    finish(0.f);
    zero_fill();
    return;
  }
  const double lse = soft_lse(all);
  const bool has_rest = rest.s != 0.f;
  const double rest_lq = has_rest ? soft_lse(rest) - lse : 0.0;
  const double rest_q = has_rest ? double(rest.s) / double(all.s) * exp2(double(rest.o) - double(all.o)) : 0.0;
  double scale_p = 1.0, rest_p = 0.0, total = 1.0, lnorm = 0.0;
  if (a.tail == AERO_TAIL_RENORM) {
    scale_p = 1.0 / mass;
    lnorm = log(mass);
  } else {
    if (has_rest) rest_p = fmax(0.0, 1.0 - mass);
    total = mass + rest_p;
  }
  double part = 0.0;
  if (there) {
    if (own_p != 0.0) part = own_p * scale_p * (own_lp - lnorm - ((own_z <= kMasked ? -INFINITY : double(own_z)) - lse));
    list.p[tid] = float(double(w) * double(a.grad_scale) * own_p * scale_p);
  }
  part = block_sum_d<NT>(part, s_dbl);   // its barriers: list.p is written
  if (rest_p > 0.0) part += rest_p * (log(rest_p) - rest_lq);
  finish(float(part));
  if (!drow) return;

  // ---- gradient row ----
  // The others' coefficient is taken relative to their own softmax, (P - p_r / q_r) q_j = (P q_r - p_r) q_j / q_r, so that it
  // stays bounded however little mass they have.
  const double g = double(w) * double(a.grad_scale);
  const float at_listed = float(g * total / double(all.s));
  const float at_other = has_rest ? float(g * (total * rest_q - rest_p) / double(rest.s)) : 0.f;
  int listed = next_listed(list, -1);
  auto turn = [&](const u32x4_t& v, int i) {
    float z[E], d[E];
    View::unpack(v, z);
#pragma unroll
    for (int e = 0; e < E; ++e) d[e] = at_other * exp2_fast(fmaf(z[e], kLog2e, -rest.o));
    if (__builtin_amdgcn_ballot_w64(i == listed) != 0 && i == listed) {
      for (int k = list.head[tid]; k >= 0; k = list.next[k])
        if (list.vec[k] == i) {
          const int own = list.elt[k];
          const float p = list.p[k];
#pragma unroll
          for (int e = 0; e < E; ++e) d[e] = e == own ? fmaf(at_listed, exp2_fast(fmaf(z[e], kLog2e, -all.o)), -p) : d[e];
        }
      listed = next_listed(list, i);
    }
    put(i, d);
  };
  const float zr = jr >= 0 ? row.at(jr) : 0.f;
  int i = tid;
  for (; i + (kAhead - 1) * NT < nvec; i += kAhead * NT) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = row.load(i + u * NT);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) turn(v[u], i + u * NT);
  }
  for (; i < nvec; i += NT) turn(row.load(i), i);
  if (jr >= 0) {
    float d = at_other * exp2_fast(fmaf(zr, kLog2e, -rest.o));
    if (listed == nvec)
      for (int k = list.head[tid]; k >= 0; k = list.next[k])
        if (list.vec[k] == nvec) d = fmaf(at_listed, exp2_fast(fmaf(zr, kLog2e, -all.o)), -list.p[k]);
    store_elt<DT>(drow, jr, d);
  }
}

// Fixed order, 64-bit sums.
constexpr int kSumNT = 1024;
__global__ __launch_bounds__(kSumNT) void k_distill_sum(const float* __restrict__ term, int64_t T, float* __restrict__ loss) {
  __shared__ double lds[kSumNT / kWave];
  constexpr int kAhead = 8;
  double acc = 0.0;
  for (int64_t t0 = threadIdx.x; t0 < T; t0 += kAhead * kSumNT) {
    float x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = t0 + u * kSumNT < T ? term[t0 + u * kSumNT] : 0.f;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) acc += double(x[u]);
  }
  acc = block_sum_d<kSumNT>(acc, lds);
  if (threadIdx.x == 0) loss[0] = float(acc);
}

size_t distill_workspace_bytes(int64_t T, int32_t V) {
  (void)V;
  return (size_t(T) * 4 + 255) / 256 * 256 + 256;
}

template <int DT, bool VEC> static void distill_launch(const DistillArgs& a, hipStream_t s) {
  const int nvec = a.V / RowView<DT, VEC>::E;
  if (nvec <= 4 * 256) hipLaunchKernelGGL((k_distill_row<256, DT, VEC>), dim3(unsigned(a.T)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_distill_row<512, DT, VEC>), dim3(unsigned(a.T)), dim3(512), 0, s, a);
}

}  // namespace aero

extern "C" aero_status aero_distill_loss_bwd(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                             const int32_t* teacher_index, const float* teacher_logprob, int32_t K,
                                             const float* token_weight, int32_t tail, float grad_scale, float* loss, float* row_loss,
                                             void* dlogits, int32_t* err_flag, void* workspace, size_t workspace_bytes,
                                             void* stream) {
  using namespace aero;
  if (T < 0 || V < 1 || V > (1 << 24) || ld < V || K < 1 || !grid_fits(T, 1024)) return AERO_ERR_SHAPE;
  if (K > kListMax) return AERO_ERR_LIMIT;
  if (tail != AERO_TAIL_RENORM && tail != AERO_TAIL_BUCKET) return AERO_ERR_SHAPE;
  if (grad_scale != grad_scale) return AERO_ERR_SHAPE;
  if (!storage_dtype_ok(dtype)) return AERO_ERR_DTYPE;
  if (!loss) return AERO_ERR_NULL;
  if (T > 0 && (!logits || !teacher_index || !teacher_logprob || !token_weight)) return AERO_ERR_NULL;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < distill_workspace_bytes(T, V))
    return AERO_ERR_WORKSPACE;
  const hipStream_t s = as_stream(stream);
  const DistillArgs a{logits, T, V, ld, teacher_index, teacher_logprob, K, token_weight, tail, grad_scale,
                      reinterpret_cast<float*>(workspace), row_loss, dlogits, err_flag};
  if (T > 0) {
    const bool vec = rows_alike(logits, dlogits, storage_bytes(dtype));
    switch (dtype) {
      case AERO_BF16: vec ? distill_launch<kBF16, true>(a, s) : distill_launch<kBF16, false>(a, s); break;
      case AERO_F16: vec ? distill_launch<kF16, true>(a, s) : distill_launch<kF16, false>(a, s); break;
      case AERO_F8E4M3: vec ? distill_launch<kF8, true>(a, s) : distill_launch<kF8, false>(a, s); break;
      default: vec ? distill_launch<kF32, true>(a, s) : distill_launch<kF32, false>(a, s);
    }
  }
  hipLaunchKernelGGL(k_distill_sum, dim3(1), dim3(kSumNT), 0, s, a.term, T, loss);
  return launch_status();
}
