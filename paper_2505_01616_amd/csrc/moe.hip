// Routing of tokens to experts, its gradient, and the dispatch of the routed
// tokens: who sits in which slot of which expert, and how many bytes every
// rank sends to every other one (the matrix of netsim_add_all_to_all).
#include <math.h>

#include "ops.h"

namespace netsim_ops {
namespace {

constexpr int kMaxExperts = 1024, kMaxTopK = 32, kMaxRanks = 1024;
constexpr float kNone = -INFINITY;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

struct Router {
  int experts, top_k, groups, kept, best;
  bool softmax, renorm;
  float scale;
};

// ---------------------------------------------------------------- routing
// A wave per row.  A lane holds the logits lane, lane + 64, ... of its row;
// every choice is the largest value of the wave, the lowest expert among
// equal ones, and is then taken out.
template <class T>
__global__ __launch_bounds__(256) void route_kernel(Router r, int64_t tokens, const T* __restrict__ logits, int64_t ld,
                                                    const float* __restrict__ bias, int32_t* __restrict__ experts,
                                                    float* __restrict__ weights) {
  extern __shared__ float shared[];
  constexpr int N = kMaxExperts / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= tokens) return;
  const T* x_row = logits + row * ld;
  const bool by_score = bias || r.best > 1;  // else the logits give the same order

  float x[N], top = kNone;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * 64 + lane;
    x[i] = e < r.experts ? (float)x_row[e] : kNone;
    bad |= isnan(x[i]) || (r.softmax && x[i] == INFINITY);
    top = fmaxf(top, x[i]);
  }
  top = wave_max(top);
  const float base = top == kNone ? 0.0f : top;
  float z = 1.0f;
  if (r.softmax && (by_score || !r.renorm)) {
    z = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) z += expf(x[i] - base);
    z = wave_sum(z);
  }

  float c[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * 64 + lane;
    c[i] = x[i];
    if (by_score && x[i] > kNone) {
      c[i] = r.softmax ? expf(x[i] - base) / z : sigmoid(x[i]);
      if (bias) c[i] += bias[e];
      bad |= isnan(c[i]);
    }
  }

  if (r.groups > 1) {
    float* row_c = shared + wave * (r.experts + 2 * r.groups);
    float* score = row_c + r.experts;
    float* keep = score + r.groups;
    const int size = r.experts / r.groups;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * 64 + lane < r.experts) row_c[i * 64 + lane] = c[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int g = lane; g < r.groups; g += 64) {
      float a = kNone, b = kNone;  // the two largest
      for (int i = 0; i < size; ++i) {
        const float v = row_c[g * size + i];
        b = v > a ? a : fmaxf(b, v);
        a = fmaxf(a, v);
      }
      score[g] = r.best > 1 && b > kNone ? a + b : a;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int g = lane; g < r.groups; g += 64) {
      const float mine = score[g];
      int before = 0;
      for (int h = 0; h < r.groups; ++h) before += score[h] > mine || (score[h] == mine && h < g);
      keep[g] = before < r.kept ? 1.0f : 0.0f;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * 64 + lane;
      if (e < r.experts && keep[e / size] == 0.0f) c[i] = kNone;
    }
  }

  const bool row_bad = __any(bad);
  int mine = -1;  // lane j keeps the j-th choice
  for (int j = 0; j < r.top_k; ++j) {
    float v = kNone;
    int at = kMaxExperts;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c[i] > v) {
        v = c[i];
        at = i * 64 + lane;
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float w = __shfl_xor(v, o, 64);
      const int b = __shfl_xor(at, o, 64);
      if (w > v || (w == v && b < at)) {
        v = w;
        at = b;
      }
    }
    if (v == kNone || row_bad) break;
    if (lane == j) mine = at;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * 64 + lane == at) c[i] = kNone;
  }

  float w = 0.0f;
  if (mine >= 0) {
    const float l = (float)x_row[mine];
    w = r.softmax ? expf(l - base) : sigmoid(l);
  }
  if (r.renorm) {
    if (r.softmax) {  // from the largest chosen logit: the sum is 1 or more
      const float l = mine >= 0 ? (float)x_row[mine] : kNone;
      const float m = wave_max(l);
      w = mine >= 0 ? expf(l - m) : 0.0f;
    }
    const float sum = wave_sum(w);
    w = sum > 0.0f ? w / sum : 0.0f;
  } else if (r.softmax) {
    w /= z;
  }
  if (lane < r.top_k) {
    experts[row * r.top_k + lane] = mine;
    weights[row * r.top_k + lane] = row_bad ? NAN : mine >= 0 ? w * r.scale : 0.0f;
  }
}

// --------------------------------------------------------- routing's gradient
// With p_j the chosen scores and w_j = scale p_j / Z (Z their sum, or 1):
//   dp_j = scale (dw_j - sum_i dw_i p_i / Z) / Z   (without the sum if Z = 1)
//   sigmoid: dl_j = dp_j p_j (1 - p_j);   softmax: dl_e = p_e (dp_e - sum_j dp_j p_j)
// A wave per row; lane j holds choice j.
template <class T>
__global__ __launch_bounds__(256) void route_back_kernel(Router r, int64_t tokens, const T* __restrict__ logits,
                                                         int64_t ld, const int32_t* __restrict__ experts,
                                                         const float* __restrict__ dweights, T* __restrict__ dlogits,
                                                         int64_t ldd) {
  extern __shared__ float shared[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= tokens) return;
  const T* x_row = logits + row * ld;
  T* out = dlogits + row * ldd;
  float* d = shared + wave * r.experts;
  for (int e = lane; e < r.experts; e += 64) d[e] = 0.0f;

  int at = -1;
  float l = kNone, dw = 0.0f;
  if (lane < r.top_k) {
    at = experts[row * r.top_k + lane];
    if (at >= r.experts) at = -1;
    if (at >= 0) {
      l = (float)x_row[at];
      dw = dweights[row * r.top_k + lane] * r.scale;
    }
  }
  const bool any = __any(at >= 0);
  float base = 0.0f, z = 1.0f;
  if (r.softmax && any) {
    if (r.renorm) {  // only the chosen scores' ratios matter
      base = wave_max(l);
    } else {
      float top = kNone;
      for (int e = lane; e < r.experts; e += 64) top = fmaxf(top, (float)x_row[e]);
      base = wave_max(top);
      z = 0.0f;
      for (int e = lane; e < r.experts; e += 64) z += expf((float)x_row[e] - base);
      z = wave_sum(z);
    }
  }
  float p = 0.0f, slope = 1.0f;
  if (at >= 0) {
    if (r.softmax) {
      p = expf(l - base) / z;
    } else {
      p = sigmoid(l);
      slope = sigmoid(-l);  // 1 - p without its cancellation
    }
  }
  float dl;
  if (r.renorm) {
    const float sum = wave_sum(p), w = sum > 0.0f ? p / sum : 0.0f;
    const float mean = wave_sum(dw * w);
    dl = w * (dw - mean) * slope;  // softmax: the chosen scores alone
  } else if (!r.softmax) {
    dl = dw * p * slope;
  } else {
    dl = dw;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (at >= 0) d[at] = dl;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (r.softmax && !r.renorm) {
    const float mean = wave_sum(dw * p);
    for (int e = lane; e < r.experts; e += 64)
      out[e] = any ? (T)(expf((float)x_row[e] - base) / z * (d[e] - mean)) : (T)0.0f;
  } else {
    for (int e = lane; e < r.experts; e += 64) out[e] = (T)d[e];
  }
}

// --------------------------------------------------------------- dispatch
// A stable counting sort of the choices by expert.  The choices are cut into
// chunks of whole tokens of one source rank; a wave counts its chunk's
// choices per expert (and per destination rank), a second kernel turns the
// counts into the chunk's first place within every expert, and a third puts
// every choice in its slot.
struct Plan {
  int experts, top_k, ranks;
  int64_t tokens, per_rank;   // tokens of a source rank
  int chunk_tokens;           // tokens of a chunk
  int64_t rank_chunks;        // chunks of a source rank
  int64_t chunks;
  bool once;
};

__device__ __forceinline__ void chunk_bounds(const Plan& p, int64_t chunk, int64_t* from, int64_t* to) {
  const int64_t rank = chunk / p.rank_chunks, part = chunk % p.rank_chunks;
  const int64_t end = min((rank + 1) * p.per_rank, p.tokens);
  *from = min(rank * p.per_rank + part * p.chunk_tokens, end);
  *to = min(*from + p.chunk_tokens, end);
}

__global__ __launch_bounds__(64) void dispatch_count_kernel(Plan p, const int32_t* __restrict__ experts,
                                                            int32_t* __restrict__ counts, int32_t* __restrict__ sent) {
  extern __shared__ int ints[];
  int* per_expert = ints;
  int* per_rank = ints + p.experts;
  const int lane = threadIdx.x;
  for (int i = lane; i < p.experts + p.ranks; i += 64) ints[i] = 0;
  __syncthreads();
  int64_t from, to;
  chunk_bounds(p, blockIdx.x, &from, &to);
  const int size = p.experts / p.ranks;
  for (int64_t i = from * p.top_k + lane; i < to * p.top_k; i += 64) {
    const int e = experts[i];
    if (e < 0 || e >= p.experts) continue;
    atomicAdd(&per_expert[e], 1);
    if (!sent) continue;
    bool counts_once = true;
    if (p.once)
      for (int64_t j = i - i % p.top_k; j < i; ++j) {
        const int before = experts[j];
        counts_once &= before < 0 || before >= p.experts || before / size != e / size;
      }
    if (counts_once) atomicAdd(&per_rank[e / size], 1);
  }
  __syncthreads();
  for (int e = lane; e < p.experts; e += 64) counts[(int64_t)blockIdx.x * p.experts + e] = per_expert[e];
  if (sent)
    for (int d = lane; d < p.ranks; d += 64) sent[(int64_t)blockIdx.x * p.ranks + d] = per_rank[d];
}

// A wave per expert: counts[chunk][e] becomes the sum over the chunks before.
__global__ __launch_bounds__(64) void dispatch_scan_kernel(Plan p, int32_t* __restrict__ counts,
                                                           int32_t* __restrict__ totals,
                                                           const int32_t* __restrict__ sent, double row_bytes,
                                                           double* __restrict__ traffic) {
  const int lane = threadIdx.x;
  if ((int)blockIdx.x < p.experts) {
    const int e = blockIdx.x;
    int carry = 0;
    for (int64_t c0 = 0; c0 < p.chunks; c0 += 64) {
      const int64_t c = c0 + lane;
      const int mine = c < p.chunks ? counts[c * p.experts + e] : 0;
      int sum = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(sum, o, 64);
        if (lane >= o) sum += v;
      }
      if (c < p.chunks) counts[c * p.experts + e] = carry + sum - mine;
      carry += __shfl(sum, 63, 64);
    }
    if (lane == 0) totals[e] = carry;
    return;
  }
  const int from = blockIdx.x - p.experts;  // a source rank
  for (int to = lane; to < p.ranks; to += 64) {
    int64_t rows = 0;
    for (int64_t c = 0; c < p.rank_chunks; ++c) rows += sent[(from * p.rank_chunks + c) * p.ranks + to];
    traffic[(int64_t)from * p.ranks + to] = (double)rows * row_bytes;
  }
}

__global__ __launch_bounds__(64) void dispatch_place_kernel(Plan p, const int32_t* __restrict__ experts,
                                                            const int32_t* __restrict__ counts,
                                                            const int32_t* __restrict__ totals,
                                                            int32_t* __restrict__ offsets,
                                                            int32_t* __restrict__ token_of_slot,
                                                            int32_t* __restrict__ slot_of_choice) {
  extern __shared__ int ints[];  // the next free slot of every expert
  const int lane = threadIdx.x;
  int carry = 0;
  for (int e0 = 0; e0 < p.experts; e0 += 64) {
    const int e = e0 + lane;
    const int mine = e < p.experts ? totals[e] : 0;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    if (e < p.experts) {
      const int first = carry + sum - mine;
      ints[e] = first + counts[(int64_t)blockIdx.x * p.experts + e];
      if (blockIdx.x == 0) offsets[e] = first;
    }
    carry += __shfl(sum, 63, 64);
  }
  if (blockIdx.x == 0 && lane == 0) offsets[p.experts] = carry;
  // slots that no choice fills
  for (int64_t s = carry + (int64_t)blockIdx.x * 64 + lane; s < p.tokens * p.top_k; s += (int64_t)gridDim.x * 64)
    token_of_slot[s] = -1;
  __syncthreads();
  int64_t from, to;
  chunk_bounds(p, blockIdx.x, &from, &to);
  for (int64_t i0 = from * p.top_k; i0 < to * p.top_k; i0 += 64) {
    const int64_t i = i0 + lane;
    int e = i < to * p.top_k ? experts[i] : -1;
    if (e >= p.experts || e < 0) e = -1;
    uint64_t same = __ballot(e >= 0);  // lanes with this lane's expert
    for (int bit = 0; (1 << bit) < p.experts; ++bit) {
      const uint64_t set = __ballot((e >> bit) & 1);
      same &= (e >> bit) & 1 ? set : ~set;
    }
    int slot = -1;
    if (e >= 0) {
      const int before = __popcll(same & ((1ull << lane) - 1));
      slot = ints[e] + before;
      token_of_slot[slot] = (int32_t)(i / p.top_k);
    }
    __syncthreads();
    if (e >= 0 && (same >> lane) == 1) ints[e] = slot + 1;  // the last lane of its expert
    __syncthreads();
    if (i < to * p.top_k) slot_of_choice[i] = slot;
  }
}

// A dispatch without tokens.
__global__ __launch_bounds__(256) void dispatch_nothing_kernel(int experts, int ranks, int32_t* offsets,
                                                               double* traffic) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i <= experts || i < ranks * ranks; i += gridDim.x * 256) {
    if (i <= experts) offsets[i] = 0;
    if (traffic && i < ranks * ranks) traffic[i] = 0.0;
  }
}

bool read_router(const netsim_router* in, Router* r, const char** why) {
  if (!in) return *why = "router is NULL", false;
  if (in->experts < 1 || in->experts > kMaxExperts) return *why = "experts must be 1 .. 1024", false;
  if (in->top_k < 1 || in->top_k > kMaxTopK || in->top_k > in->experts)
    return *why = "top_k must be 1 .. 32 and at most experts", false;
  if (in->scores != NETSIM_SCORES_SOFTMAX && in->scores != NETSIM_SCORES_SIGMOID) return *why = "bad scores", false;
  if (in->groups < 1 || in->experts % in->groups != 0) return *why = "groups must divide experts", false;
  if (in->groups_kept < 1 || in->groups_kept > in->groups) return *why = "groups_kept must be 1 .. groups", false;
  if (in->group_best != 1 && in->group_best != 2) return *why = "group_best must be 1 or 2", false;
  if (in->renormalise != 0 && in->renormalise != 1) return *why = "renormalise must be 0 or 1", false;
  if (!isfinite(in->scale)) return *why = "scale must be finite", false;
  *r = Router{in->experts, in->top_k, in->groups, in->groups_kept, in->groups > 1 ? in->group_best : 1,
              in->scores == NETSIM_SCORES_SOFTMAX, in->renormalise != 0, in->scale};
  return true;
}

constexpr int64_t kMaxChoices = 0x7fffffff;

// The plan of a dispatch (tokens >= 1).
Plan make_plan(int32_t experts, int32_t top_k, int64_t tokens, int32_t ranks, int64_t per_rank, bool once) {
  Plan p{};
  p.experts = experts;
  p.top_k = top_k;
  p.ranks = ranks;
  p.tokens = tokens;
  p.per_rank = per_rank < tokens ? per_rank : tokens;
  p.once = once;
  p.chunk_tokens = 1024 / top_k;
  p.rank_chunks = ceil_div(p.per_rank, p.chunk_tokens);
  p.chunks = p.rank_chunks * ranks;
  return p;
}

// The tokens' share of the checks of a dispatch and of its workspace.
const char* bad_dispatch(int32_t experts, int32_t top_k, int64_t tokens, int32_t ranks, int64_t per_rank) {
  if (experts < 1 || experts > kMaxExperts) return "experts must be 1 .. 1024";
  if (top_k < 1 || top_k > kMaxTopK) return "top_k must be 1 .. 32";
  if (ranks < 1 || ranks > kMaxRanks || experts % ranks != 0) return "ranks must be 1 .. 1024 and divide experts";
  if (tokens < 0 || tokens > kMaxChoices / top_k) return "tokens must be >= 0, with at most 2^31-1 choices";
  if (per_rank < 1 || ceil_div(tokens, per_rank) > ranks) return "tokens_per_rank must be >= 1 and hold the tokens";
  return nullptr;
}

}  // namespace
}  // namespace netsim_ops

using namespace netsim_ops;

extern "C" netsim_status netsim_route(int32_t device, const netsim_router* router, int64_t tokens, int32_t type,
                                      const void* d_logits, int64_t ld_logits, const float* d_bias,
                                      int32_t* d_experts, float* d_weights, void* hip_stream) {
  const char* what = "route";
  return entry(what, device, [&] {
    Router r;
    const char* why = "";
    if (!read_router(router, &r, &why)) return fail(NETSIM_E_INVALID, what, why);
    if (!type_ok(type)) return fail(NETSIM_E_INVALID, what, "bad type");
    if (tokens < 0 || tokens > kMaxChoices / r.top_k)
      return fail(NETSIM_E_INVALID, what, "tokens must be >= 0, with at most 2^31-1 choices");
    if (ld_logits < r.experts) return fail(NETSIM_E_INVALID, what, "ld_logits is below experts");
    if (tokens == 0) return (netsim_status)NETSIM_OK;
    if (!d_logits || !d_experts || !d_weights) return fail(NETSIM_E_INVALID, what, "NULL array");
    if (!aligned(d_logits, type_size(type)) || !aligned(d_bias, 4) || !aligned(d_experts, 4) || !aligned(d_weights, 4))
      return fail(NETSIM_E_INVALID, what, "an array is not aligned to its type");
    return launch(what, device, [&] {
      const size_t lds = r.groups > 1 ? 4 * sizeof(float) * (r.experts + 2 * r.groups) : 0;
      with_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(route_kernel<T>, dim3((unsigned)ceil_div(tokens, 4)), dim3(256), lds,
                           static_cast<hipStream_t>(hip_stream), r, tokens, static_cast<const T*>(d_logits), ld_logits,
                           d_bias, d_experts, d_weights);
      });
    });
  });
}

extern "C" netsim_status netsim_route_backward(int32_t device, const netsim_router* router, int64_t tokens,
                                               int32_t type, const void* d_logits, int64_t ld_logits,
                                               const int32_t* d_experts, const float* d_dweights, void* d_dlogits,
                                               int64_t ld_dlogits, void* hip_stream) {
  const char* what = "route_backward";
  return entry(what, device, [&] {
    Router r;
    const char* why = "";
    if (!read_router(router, &r, &why)) return fail(NETSIM_E_INVALID, what, why);
    if (!type_ok(type)) return fail(NETSIM_E_INVALID, what, "bad type");
    if (tokens < 0 || tokens > kMaxChoices / r.top_k)
      return fail(NETSIM_E_INVALID, what, "tokens must be >= 0, with at most 2^31-1 choices");
    if (ld_logits < r.experts || ld_dlogits < r.experts)
      return fail(NETSIM_E_INVALID, what, "ld_logits or ld_dlogits is below experts");
    if (tokens == 0) return (netsim_status)NETSIM_OK;
    if (!d_logits || !d_experts || !d_dweights || !d_dlogits) return fail(NETSIM_E_INVALID, what, "NULL array");
    if (!aligned(d_logits, type_size(type)) || !aligned(d_dlogits, type_size(type)) || !aligned(d_experts, 4) ||
        !aligned(d_dweights, 4))
      return fail(NETSIM_E_INVALID, what, "an array is not aligned to its type");
    return launch(what, device, [&] {
      with_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(route_back_kernel<T>, dim3((unsigned)ceil_div(tokens, 4)), dim3(256),
                           4 * sizeof(float) * r.experts, static_cast<hipStream_t>(hip_stream), r, tokens,
                           static_cast<const T*>(d_logits), ld_logits, d_experts, d_dweights,
                           static_cast<T*>(d_dlogits), ld_dlogits);
      });
    });
  });
}

extern "C" int64_t netsim_dispatch_work_bytes(int32_t experts, int32_t top_k, int64_t tokens, int32_t ranks,
                                              int64_t tokens_per_rank) {
  if (bad_dispatch(experts, top_k, tokens, ranks, tokens_per_rank)) return -1;
  if (tokens == 0) return 0;
  const Plan p = make_plan(experts, top_k, tokens, ranks, tokens_per_rank, false);
  return 4 * (p.chunks * (p.experts + p.ranks) + p.experts);
}

extern "C" netsim_status netsim_dispatch(int32_t device, int32_t experts, int32_t top_k, int64_t tokens,
                                         const int32_t* d_experts, int32_t ranks, int64_t tokens_per_rank,
                                         double row_bytes, int32_t once_per_rank, int32_t* d_offsets,
                                         int32_t* d_token_of_slot, int32_t* d_slot_of_choice, double* d_traffic,
                                         void* d_work, int64_t work_bytes, void* hip_stream) {
  const char* what = "dispatch";
  return entry(what, device, [&] {
    if (const char* why = bad_dispatch(experts, top_k, tokens, ranks, tokens_per_rank))
      return fail(NETSIM_E_INVALID, what, why);
    if (!(row_bytes >= 0) || !isfinite(row_bytes))
      return fail(NETSIM_E_INVALID, what, "row_bytes must be finite and >= 0");
    if (once_per_rank != 0 && once_per_rank != 1) return fail(NETSIM_E_INVALID, what, "once_per_rank must be 0 or 1");
    if (!d_offsets || (tokens > 0 && (!d_experts || !d_token_of_slot || !d_slot_of_choice)))
      return fail(NETSIM_E_INVALID, what, "NULL array");
    if (work_bytes < netsim_dispatch_work_bytes(experts, top_k, tokens, ranks, tokens_per_rank) ||
        (tokens > 0 && !d_work))
      return fail(NETSIM_E_INVALID, what, "the workspace is too small (netsim_dispatch_work_bytes)");
    if (!aligned(d_experts, 4) || !aligned(d_offsets, 4) || !aligned(d_token_of_slot, 4) ||
        !aligned(d_slot_of_choice, 4) || !aligned(d_traffic, 8) || !aligned(d_work, 4))
      return fail(NETSIM_E_INVALID, what, "an array is not aligned to its type");
    const Plan p = make_plan(experts, top_k, tokens > 0 ? tokens : 1, ranks, tokens_per_rank, once_per_rank != 0);
    return launch(what, device, [&] {
      hipStream_t s = static_cast<hipStream_t>(hip_stream);
      if (tokens == 0) {
        hipLaunchKernelGGL(dispatch_nothing_kernel, dim3(64), dim3(256), 0, s, experts, ranks, d_offsets, d_traffic);
        return;
      }
      int32_t* counts = static_cast<int32_t*>(d_work);
      int32_t* sent = counts + p.chunks * p.experts;
      int32_t* totals = sent + p.chunks * p.ranks;
      hipLaunchKernelGGL(dispatch_count_kernel, dim3((unsigned)p.chunks), dim3(64), sizeof(int) * (experts + ranks), s,
                         p, d_experts, counts, d_traffic ? sent : nullptr);
      hipLaunchKernelGGL(dispatch_scan_kernel, dim3(experts + (d_traffic ? ranks : 0)), dim3(64), 0, s, p, counts,
                         totals, sent, row_bytes, d_traffic);
      hipLaunchKernelGGL(dispatch_place_kernel, dim3((unsigned)p.chunks), dim3(64), sizeof(int) * experts, s, p,
                         d_experts, counts, totals, d_offsets, d_token_of_slot, d_slot_of_choice);
    });
  });
}
