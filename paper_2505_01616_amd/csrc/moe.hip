// Routing of tokens to experts, its gradient, and the dispatch of the routed
// tokens: who sits in which slot of which expert, and how many bytes every
// rank sends to every other one (the matrix of netsim_add_all_to_all).
#include <math.h>

#include <type_traits>

#include "ops.h"

namespace netsim_ops {
namespace {

constexpr int kMaxExperts = 1024, kMaxTopK = 32, kMaxRanks = 1024;
constexpr float kNone = -INFINITY;

// ------------------------------------------------ exchanges between L lanes
// L = 8, 16 or 64 neighbouring lanes hold a row.  Exchanges inside 16 lanes
// are register moves; over a whole wave the last lane holds the result and
// is read from there.  Every lane ends up with the result, and sums are
// formed in the same order everywhere.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int old, int v) {
  // with all rows taking part every lane has a partner, and the move can be
  // part of the instruction that uses it
  return __builtin_amdgcn_update_dpp(ROWS == 0xF ? 0 : old, v, CTRL, ROWS, 0xF, ROWS == 0xF);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float old, float v) {
  return __int_as_float(moved<CTRL, ROWS>(__float_as_int(old), __float_as_int(v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double old, double v) {
  const long long o = __double_as_longlong(old), b = __double_as_longlong(v);
  const int lo = moved<CTRL, ROWS>((int)o, (int)b), hi = moved<CTRL, ROWS>((int)(o >> 32), (int)(b >> 32));
  return __longlong_as_double((long long)hi << 32 | (unsigned)lo);
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ float last_lane(float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63)); }
__device__ __forceinline__ double last_lane(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_readlane((int)b, 63), hi = __builtin_amdgcn_readlane((int)(b >> 32), 63);
  return __longlong_as_double((long long)hi << 32 | (unsigned)lo);
}
// old(v): what a lane without a partner combines with.
template <int L, class V, class Old, class Op>
__device__ __forceinline__ V over(V v, Old old, Op op) {
  v = op(v, moved<0xB1, 0xF>(old(v), v));   // 1 lane apart
  v = op(v, moved<0x4E, 0xF>(old(v), v));   // 2 apart
  v = op(v, moved<0x141, 0xF>(old(v), v));  // mirrored in 8 lanes
  if constexpr (L > 8) v = op(v, moved<0x140, 0xF>(old(v), v));  // mirrored in 16
  if constexpr (L > 16) {
    v = op(v, moved<0x142, 0xA>(old(v), v));  // the last lane of the 16 before
    v = op(v, moved<0x143, 0xC>(old(v), v));  // lane 31
    v = last_lane(v);
  }
  return v;
}
template <int L>
__device__ __forceinline__ float max_over(float v) {
  return over<L>(v, [](float x) { return x; }, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ __forceinline__ float sum_over(float v) {
  return over<L>(v, [](float) { return 0.0f; }, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ bool any_over(bool v) {
  const uint64_t set = __ballot(v);
  if constexpr (L == 64)
    return set != 0;
  else
    return (set >> (threadIdx.x & 63 & ~(L - 1)) & ((1ull << L) - 1)) != 0;
}

// exp(x) to about two units in the last place: 2^(x log2 e) with the part of
// the product that 32 bits cut off put back.
__device__ __forceinline__ float exp_of(float x) {
  constexpr float LOG2E = 1.44269504088896340736f, LOG2E_LOW = 1.925963033500e-8f, LN2 = 0.69314718055994530942f;
  const float hi = x * LOG2E;
  const float low = __builtin_fmaf(x, LOG2E_LOW, __builtin_fmaf(x, LOG2E, -hi));
  const float p = __builtin_amdgcn_exp2f(hi);
  // From 128 on p is infinite, which a low of 0 or less would turn into a NaN;
  // below -128 it is 0 or nearly so.  Neither takes a correction, and low may
  // not be finite there.
  return fabsf(hi) < 128.0f ? __builtin_fmaf(p, low * LN2, p) : p;
}
// exp(x) for x <= 0 with the product rounded: off by |x| half steps more.  For
// softmax's sum alone, where what is far away counts little: 1,023 of 1,024
// logits 5 below the largest, the worst case, leave weights off by 4.1 units
// in the last place (2.2 with exp_of, which takes 262,144 rows of 128 from 27.7
// to 30.0 us); in ordinary rows both leave the 7.6 that float32 logits'
// differences are rounded by.
__device__ __forceinline__ float exp_near(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }
// To 1.8 units in the last place; 1.5 with the quotient refined, which takes
// 16,384 rows of 256 from 13.6 to 14.1 us.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }

struct Router {
  int experts, top_k, groups, kept, best;
  bool softmax, renorm;
  float scale;
};

// N values of a row in each of L lanes, in vectors of V neighbouring ones:
// value i of lane j is element (i / V * L + j) * V + i % V.
template <class T, int L, int N>
struct Row {
  static constexpr int V = N < (int)(16 / sizeof(T)) ? N : (int)(16 / sizeof(T));
  static __device__ __forceinline__ int element(int i, int j) { return (i / V * L + j) * V + i % V; }
  struct alignas(V * sizeof(T)) Vector {
    T v[V];
  };
  // Places beyond the row hold minus infinity.  wide: every vector lies
  // wholly inside or outside the row, and is aligned.
  static __device__ __forceinline__ void load(const T* row, int n, int j, bool wide, Vector (&in)[N / V], float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N / V; ++i) {
      const int e = element(i * V, j);
#pragma unroll
      for (int h = 0; h < V; ++h) in[i].v[h] = (T)kNone;
      if (wide) {
        if (e < n) in[i] = *reinterpret_cast<const Vector*>(row + e);
      } else {
#pragma unroll
        for (int h = 0; h < V; ++h)
          if (e + h < n) in[i].v[h] = row[e + h];
      }
#pragma unroll
      for (int h = 0; h < V; ++h) x[i * V + h] = (float)in[i].v[h];
    }
  }
};

// ---------------------------------------------------------------- routing
// L lanes per row, N logits each, in registers; one pass over the logits.
//
// A choice value and its expert make one key, so that a compare-and-exchange
// is a minimum and a maximum: of equal values the lowest expert is the
// largest key.  Each lane sorts its keys; the largest of a row is the
// largest of the lanes' first ones, and the lane that gave it moves on to
// its next.
//
// Bound by instructions per row: few lanes per row mean few exchanges (8
// lanes: three per choice, eight rows at once), many lanes mean short sorts
// and enough waves where rows are few.  262,144 rows of 128 bfloat16 logits,
// six choices: 27 us (2.9 TB/s), 507 vector instructions per eight rows, 16 of
// them exponentials at a quarter of the rate: 31,000 cycles of each SIMD.
// 16,384 rows of 256 float32 logits, sigmoid scores, a bias and groups: 14 us,
// 1,279 instructions per four rows, 9 us of it, with four waves a SIMD to hide
// the groups' passes through shared memory (131,072 rows: 70 us).

// A 32-bit value in a 64-bit float leaves its low 29 bits free.
struct WideKey {
  using type = double;
  static constexpr double NONE = -0x1p996;    // below every value; infinities move to +-2^996
  static __device__ __forceinline__ double larger(double a, double b) {
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));   // keys are never NaN
    return r;
  }
  static __device__ __forceinline__ double smaller(double a, double b) {
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
  }
  static __device__ __forceinline__ double of(float value, int expert) {
    // + 0: -0 is 0
    const long long b = __double_as_longlong(larger(smaller((double)(value + 0.0f), 0x1p996), NONE));
    const int hi = (int)(b >> 32), low = (expert ^ (kMaxExperts - 1)) ^ ((hi >> 31) & (kMaxExperts - 1));
    return __longlong_as_double((b & ~0x1FFFFFFFll) | low);
  }
  static __device__ __forceinline__ int expert(double key) {
    const long long b = __double_as_longlong(key);
    const int low = (int)b & (kMaxExperts - 1);
    return key <= NONE ? -1 : b < 0 ? low : low ^ (kMaxExperts - 1);
  }
};
// Values of 16 bits in their order as signed whole numbers (-0 is 0), above
// the expert.
template <class T>
struct ShortKey {
  using type = int32_t;
  static constexpr int32_t NONE = INT32_MIN;
  typedef short pair __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ int32_t larger(int32_t a, int32_t b) { return a > b ? a : b; }
  static __device__ __forceinline__ int32_t smaller(int32_t a, int32_t b) { return a > b ? b : a; }
  // The keys of two neighbouring values, their bits in one word.
  static __device__ __forceinline__ void of(uint32_t bits, int expert, int32_t* first, int32_t* second) {
    const pair b = __builtin_bit_cast(pair, bits), sign = b >> (short)15;
    const uint32_t order = __builtin_bit_cast(uint32_t, (pair)((b ^ (sign & (short)0x7FFF)) - sign));
    *first = (int32_t)(order << 16 | (uint32_t)(kMaxExperts - 1 - expert));
    *second = (int32_t)((order & 0xFFFF0000u) | (uint32_t)(kMaxExperts - 2 - expert));
  }
  static __device__ __forceinline__ int expert(int32_t key) {
    constexpr int INF = std::is_same_v<T, bf16> ? 0x7F80 : 0x7C00;   // of minus infinity: -INF
    return (key >> 16) > -INF ? kMaxExperts - 1 - (key & 0xFFFF) : -1;
  }
};

template <class Key, class K>
__device__ __forceinline__ void exchange(K& a, K& b) {
  const K more = Key::larger(a, b), less = Key::smaller(a, b);
  a = more;
  b = less;
}
// Descending order of FROM .. FROM + N - 1 by odd-even merges (Batcher 1968).
template <class Key, int FROM, int N, class K, int SIZE>
__device__ __forceinline__ void sort_keys(K (&k)[SIZE]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int h = p; h >= 1; h /= 2)
#pragma unroll
      for (int j = h % p; j + h < N; j += 2 * h)
#pragma unroll
        for (int i = 0; i < h; ++i)
          if (i + j + h < N && (i + j) / (2 * p) == (i + j + h) / (2 * p))
            exchange<Key>(k[FROM + i + j], k[FROM + i + j + h]);
}
// The M largest of N keys in descending order, in k[0 .. M-1].
template <class Key, int M, class K, int N>
__device__ __forceinline__ void largest_keys(K (&k)[N]) {
  if constexpr (M == N) {
    sort_keys<Key, 0, N>(k);
  } else {
    static_assert(N == 2 * M, "two lists are merged");
    sort_keys<Key, 0, M>(k);
    sort_keys<Key, M, M>(k);
    // the larger of each pair from the two ends rises and falls once
#pragma unroll
    for (int i = 0; i < M; ++i) k[i] = Key::larger(k[i], k[N - 1 - i]);
#pragma unroll
    for (int h = M / 2; h >= 1; h /= 2)
#pragma unroll
      for (int i = 0; i < M; ++i)
        if ((i & h) == 0) exchange<Key>(k[i], k[i + h]);
  }
}

// FEW: top_k <= 8.  BY_SCORE: scores are compared, not logits.
template <class T, int L, int N, bool FEW, bool BY_SCORE>
__global__ __launch_bounds__(256) void route_kernel(Router r, int64_t tokens, const T* __restrict__ logits, int64_t ld,
                                                    bool wide, const float* __restrict__ bias,
                                                    int32_t* __restrict__ experts, float* __restrict__ weights) {
  extern __shared__ float shared[];
  using R = Row<T, L, N>;
  constexpr bool SHORT = sizeof(T) == 2 && !BY_SCORE;
  using Key = std::conditional_t<SHORT, ShortKey<T>, WideKey>;
  using K = typename Key::type;
  constexpr int M = FEW && N > 8 ? 8 : N, SLOTS = FEW ? 1 : (kMaxTopK + L - 1) / L;
  const int j = threadIdx.x & (L - 1);
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const int64_t row = at < tokens ? at : tokens - 1;   // lanes beyond repeat the last row and write nothing
  const T* x_row = logits + row * ld;

  float x[N], add[N], top = kNone;
  typename R::Vector in[N / R::V];
  R::load(x_row, r.experts, j, wide, in, x);
  if constexpr (BY_SCORE)   // here, where nothing waits for it yet
#pragma unroll
    for (int i = 0; i < N; ++i) add[i] = bias && R::element(i, j) < r.experts ? bias[R::element(i, j)] : 0.0f;
  // a NaN, and plus infinity under softmax, make the scores or their sum NaN;
  // where neither is formed the logits are looked at
  bool bad = false;
  const bool sum_all = r.softmax && (BY_SCORE || !r.renorm);
  if (!BY_SCORE && !sum_all) {
    const int undefined = r.softmax ? 0x203 : 0x003;
#pragma unroll
    for (int i = 0; i < N; ++i) bad |= __builtin_amdgcn_classf(x[i], undefined);
  }
  float base = 0.0f, z = 1.0f;
  if (sum_all) {
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, x[i]);
    top = max_over<L>(top);
    base = top == kNone ? 0.0f : top;
    z = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) z += exp_near(x[i] - base);
    z = sum_over<L>(z);
    bad = isnan(z);
  }
  if constexpr (BY_SCORE) {
    const float inverse = 1.0f / z;
    float c[N];
    if (r.softmax) {
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = exp_of(x[i] - base) * inverse;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = sigmoid(x[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float value = c[i] + add[i];
      bad |= x[i] != kNone && isnan(value);
      x[i] = x[i] == kNone ? kNone : value;
    }
  }

  if (r.groups > 1) {
    // the row's choice values in shared memory; as many lanes as there are
    // for each group look through its members
    const int size = r.experts / r.groups;
    constexpr int pitch = L * N + 1;   // places beyond the experts hold minus infinity
    float* row_c = shared + (threadIdx.x / L) * (pitch + 2 * r.groups);
    float* score = row_c + pitch;
    float* keep = score + r.groups;
#pragma unroll
    for (int i = 0; i < N; ++i) row_c[R::element(i, j)] = x[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int share = 1;   // lanes of a group, a power of two
    while (2 * share * r.groups <= L) share *= 2;
    for (int g0 = 0; g0 < r.groups; g0 += L / share) {
      const int g = g0 + j / share;
      const float* member = row_c + (g < r.groups ? g : 0) * size;
      float a = kNone, b = kNone;  // the two largest
#pragma unroll 4
      for (int i = j & (share - 1); i < size; i += share) {
        const float v = member[i];
        b = fmaxf(b, fminf(a, v));
        a = fmaxf(a, v);
      }
      for (int o = 1; o < share; o *= 2) {
        const float a2 = __shfl_xor(a, o, 64), b2 = __shfl_xor(b, o, 64);
        b = fmaxf(fmaxf(b, b2), fminf(a, a2));
        a = fmaxf(a, a2);
      }
      if (g < r.groups && (j & (share - 1)) == 0) score[g] = r.best > 1 && b > kNone ? a + b : a;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int g = j; g < r.groups; g += L) {
      const float mine = score[g];
      int before = 0;
#pragma unroll 4
      for (int h = 0; h < r.groups; ++h) before += score[h] > mine || (score[h] == mine && h < g);
      keep[g] = before < r.kept ? 1.0f : 0.0f;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const float per = 1.0f / size;
    const bool aligned = size % R::V == 0;   // a vector lies in one group
#pragma unroll
    for (int i = 0; i < N; i += R::V) {
      float kept = 1.0f;
#pragma unroll
      for (int h = 0; h < R::V; ++h) {
        const int e = R::element(i + h, j);
        // (e + 1/2) / size in 32 bits is never off by half a step below 2^10
        if (h == 0 || !aligned) kept = keep[min((int)((e + 0.5f) * per), r.groups - 1)];
        x[i + h] = kept == 0.0f ? kNone : x[i + h];
      }
    }
  }

  K k[N];
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    if constexpr (SHORT) {
      uint32_t bits;
      __builtin_memcpy(&bits, &in[i / R::V].v[i % R::V], 4);
      Key::of(bits, R::element(i, j), &k[i], &k[i + 1]);
    } else {
      k[i] = Key::of(x[i], R::element(i, j));
      k[i + 1] = Key::of(x[i + 1], R::element(i + 1, j));
    }
  }
  if (SHORT && r.groups > 1)
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = x[i] == kNone ? Key::NONE : k[i];
  largest_keys<Key, M>(k);
  int mine[SLOTS];  // lane j keeps the choices j, j + L, ...
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) mine[s] = -1;
  for (int c = 0; c < r.top_k; ++c) {
    const K best = over<L>(k[0], [](K v) { return v; }, [](K a, K b) { return Key::larger(a, b); });
    const bool taken = k[0] == best;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const K here = k[i], after = i + 1 < M ? k[i + 1] : Key::NONE;   // values: an index chosen at run time costs M selects
      k[i] = taken ? after : here;
    }
    const int expert = Key::expert(best);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s)
      if (c == s * L + j) mine[s] = expert;
  }

  const bool row_bad = any_over<L>(bad);
  float l[SLOTS], w[SLOTS], sum = 0.0f, most = kNone;
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    l[s] = mine[s] >= 0 ? (float)x_row[mine[s]] : kNone;
    most = fmaxf(most, l[s]);
  }
  // renormalised softmax from the largest chosen logit: the sum is 1 or more
  if (r.softmax && r.renorm) base = max_over<L>(most);
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    w[s] = mine[s] < 0 ? 0.0f : r.softmax ? exp_of(l[s] - base) : sigmoid(l[s]);
    sum += w[s];
  }
  if (r.renorm) z = sum_over<L>(sum);
#pragma unroll
  for (int s = 0; s < SLOTS; ++s)
    if (at < tokens && s * L + j < r.top_k) {
      const int64_t to = row * r.top_k + s * L + j;
      experts[to] = row_bad ? -1 : mine[s];
      // divided first: scale / z may be infinite where the weight is not
      weights[to] = row_bad ? NAN : z > 0.0f ? w[s] / z * r.scale : 0.0f;
    }
}

// --------------------------------------------------------- routing's gradient
// With p_j the chosen scores and w_j = scale p_j / Z (Z their sum, or 1):
//   dp_j = scale (dw_j - sum_i dw_i p_i / Z) / Z   (without the sum if Z = 1)
//   sigmoid: dl_j = dp_j p_j (1 - p_j);   softmax: dl_e = p_e (dp_e - sum_j dp_j p_j)
// With renormalised scores softmax's last sum is 0, so there, and for
// sigmoid, only the chosen logits matter: only they are read, and the rest
// of a row is zeros.
struct Chosen {
  int at;         // the expert, -1 for none
  float l, dw;    // its logit, and its weight's gradient times scale
};
template <class T>
__device__ __forceinline__ Chosen choice(const Router& r, const T* x_row, const int32_t* experts, const float* dweights,
                                         int64_t row, int c) {
  Chosen out{-1, kNone, 0.0f};
  if (c < r.top_k) {
    const int e = experts[row * r.top_k + c];
    if (e >= 0 && e < r.experts) out = Chosen{e, (float)x_row[e], dweights[row * r.top_k + c] * r.scale};
  }
  return out;
}

// Only the chosen logits: K lanes per row, K >= top_k, 64 / K rows per wave.
// Gradients are scattered into a row of shared memory, from where the wave
// writes its rows as vectors.  Bound by the rows written: 131,072 rows of 256
// float32 gradients, eight choices, take 35 us (134 MB written, 3.9 TB/s),
// 48 us where the lines of the chosen logits come from memory and not from
// the last cache.
template <class T, int K>
__global__ __launch_bounds__(256) void route_back_chosen_kernel(Router r, int64_t tokens, const T* __restrict__ logits,
                                                                int64_t ld, const int32_t* __restrict__ experts,
                                                                const float* __restrict__ dweights,
                                                                T* __restrict__ dlogits, int64_t ldd, bool wide) {
  extern __shared__ float shared[];
  constexpr int ROWS = 64 / K, V = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane & (K - 1);
  const int pitch = (r.experts + V - 1) / V * V;
  float* mine = shared + wave * ROWS * pitch;
  for (int i = lane * 4; i < ROWS * pitch; i += 256) *reinterpret_cast<float4*>(mine + i) = make_float4(0, 0, 0, 0);
  const int64_t first = ((int64_t)blockIdx.x * 4 + wave) * ROWS, row = first + lane / K;
  if (first >= tokens) return;
  Chosen c{-1, kNone, 0.0f};
  if (row < tokens) c = choice(r, logits + row * ld, experts, dweights, row, j);
  float p = 0.0f, slope = 1.0f;
  // lanes exchange over 8, 16 or 64: rows of 32 lanes take two steps more
  auto total = [](float v) {
    if constexpr (K == 32) {
      v = sum_over<16>(v);
      return v + __shfl_xor(v, 16, 64);
    } else {
      return sum_over<K>(v);
    }
  };
  if (r.softmax) {
    float base = c.l;
    if constexpr (K == 32) {
      base = max_over<16>(base);
      base = fmaxf(base, __shfl_xor(base, 16, 64));
    } else {
      base = max_over<K>(base);
    }
    if (c.at >= 0) p = exp_of(c.l - base);
  } else if (c.at >= 0) {
    p = sigmoid(c.l);
    slope = sigmoid(-c.l);  // 1 - p without its cancellation
  }
  float dl = c.dw * p * slope;
  if (r.renorm) {
    const float sum = total(p), w = sum > 0.0f ? p / sum : 0.0f;
    dl = w * (c.dw - total(c.dw * w)) * slope;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (c.at >= 0) mine[lane / K * pitch + c.at] = dl;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int rows = (int)(tokens - first < ROWS ? tokens - first : ROWS);
  if (wide) {
    const int vectors = r.experts / V;
    for (int i = lane; i < rows * vectors; i += 64) {
      const int line = i / vectors, e = (i - line * vectors) * V;
      struct alignas(16) Vector {
        T v[V];
      } out;
#pragma unroll
      for (int h = 0; h < V; ++h) out.v[h] = (T)mine[line * pitch + e + h];
      *reinterpret_cast<Vector*>(dlogits + (first + line) * ldd + e) = out;
    }
  } else {
    for (int line = 0; line < rows; ++line)
      for (int e = lane; e < r.experts; e += 64) dlogits[(first + line) * ldd + e] = (T)mine[line * pitch + e];
  }
}

// Softmax without renormalisation: every logit of a row has a gradient.  The
// row in registers as for routing; the chosen ones' dp through shared memory.
// Bound by memory: 65,536 rows of 128 bfloat16 logits take 10.8 us (3.1 TB/s).
template <class T, int L, int N>
__global__ __launch_bounds__(256) void route_back_kernel(Router r, int64_t tokens, const T* __restrict__ logits,
                                                         int64_t ld, bool wide, const int32_t* __restrict__ experts,
                                                         const float* __restrict__ dweights, T* __restrict__ dlogits,
                                                         int64_t ldd, bool wide_out) {
  using R = Row<T, L, N>;
  constexpr int SLOTS = (kMaxTopK + L - 1) / L;
  __shared__ float shared[256 * N + 256 / L];
  const int j = threadIdx.x & (L - 1);
  const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L, row = id < tokens ? id : tokens - 1;
  const T* x_row = logits + row * ld;
  float* d = shared + threadIdx.x / L * (L * N + 1);
  float x[N], top = kNone;
  typename R::Vector in[N / R::V];
  R::load(x_row, r.experts, j, wide, in, x);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    d[R::element(i, j)] = 0.0f;
    top = fmaxf(top, x[i]);
  }
  top = max_over<L>(top);
  const float base = top == kNone ? 0.0f : top;
  float z = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = exp_of(x[i] - base);
    z += x[i];
  }
  z = sum_over<L>(z);
  const float inverse = z > 0.0f ? 1.0f / z : 0.0f;
  float mean = 0.0f;
  bool any = false;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    const Chosen c = choice(r, x_row, experts, dweights, row, s * L + j);
    if (c.at >= 0) {
      d[c.at] = c.dw;
      mean += c.dw * exp_of(c.l - base) * inverse;
      any = true;
    }
  }
  mean = sum_over<L>(mean);
  any = any_over<L>(any);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (id >= tokens) return;
  T* out = dlogits + row * ldd;
#pragma unroll
  for (int i = 0; i < N; i += R::V) {
    const int e = R::element(i, j);
    struct alignas(R::V * sizeof(T)) Vector {
      T v[R::V];
    } v;
#pragma unroll
    for (int h = 0; h < R::V; ++h) v.v[h] = any ? (T)(x[i + h] * inverse * (d[e + h] - mean)) : (T)0.0f;
    if (wide_out) {
      if (e < r.experts) *reinterpret_cast<Vector*>(out + e) = v;
    } else {
#pragma unroll
      for (int h = 0; h < R::V; ++h)
        if (e + h < r.experts) out[e + h] = v.v[h];
    }
  }
}

// Calls f with the lanes per row and the values per lane as constants.
// Fewer lanes per row exchange less per row, as long as a lane holds at most
// 16 values and the rows still make 4,096 waves (4 for each of the 1,024
// SIMDs).  131,072 rows of 128 bfloat16 logits take 18 us in 8 lanes, 20 in
// 16 and 49 in 64; 16,384 rows of 256 float32 ones in groups 14 us in 16 lanes
// and 18 in 64.
template <class F>
void with_shape(int64_t tokens, int experts, F&& f) {
  int lanes = 64;
  for (int fewer : {16, 8})
    if (experts <= fewer * 16 && tokens * fewer >= 64 * 4096) lanes = fewer;
  auto values = [&](auto l) {
    constexpr int L = decltype(l)::value;
    const int n = (experts + L - 1) / L;
    if (n <= 4)
      f(l, std::integral_constant<int, 4>{});
    else if (n <= 8)
      f(l, std::integral_constant<int, 8>{});
    else
      f(l, std::integral_constant<int, 16>{});
  };
  if (lanes == 8)
    values(std::integral_constant<int, 8>{});
  else if (lanes == 16)
    values(std::integral_constant<int, 16>{});
  else
    values(std::integral_constant<int, 64>{});
}

constexpr int64_t kRowsOfLaunch = 1 << 25;   // of up to 64 threads each

// Whether vectors of V elements of every row are aligned and whole.
template <class T>
bool whole_vectors(const void* p, int64_t ld, int experts, int vector) {
  return experts % vector == 0 && ld % vector == 0 && aligned(p, vector * (int64_t)sizeof(T));
}

// --------------------------------------------------------------- dispatch
// A stable counting sort of the choices by expert.  The choices are cut into
// chunks of whole tokens of one source rank; a wave counts its chunk's
// choices per expert (and per destination rank), a second kernel turns the
// counts into the chunk's first place within every expert, and a third puts
// every choice in its slot.  Few choices take one workgroup and one launch.
// The counters are whole numbers, so the order of additions does not matter.
//
// Bound by the length of each wave's chain of ballots and counters, not by
// bytes (12.6 MB for 1,048,576 choices of 256 experts from 64 ranks): 6.8 us
// counting, 5.4 us adding up, 9.9 us placing.  Chunks of 1,024 choices make 1,024
// waves there, one for each SIMD, so nothing hides a wave's chain.  48 choices in
// one launch: 4.2 us.
struct Plan {
  int experts, top_k, ranks;
  int64_t tokens, per_rank;   // tokens of a source rank
  int chunk_tokens;           // tokens of a chunk
  int64_t rank_chunks;        // chunks of a source rank; the last that holds tokens may have fewer
  int64_t chunks;             // of the ranks that hold tokens: the first ones
  bool once;
  bool small;                 // one workgroup does it all
};
// One launch is shorter to enqueue than three: 8,192 choices of 256 experts
// take 13 us a call in one workgroup and 19 in three launches, 16,384 take 22
// and 19.
constexpr int kSmallChoices = 8192, kSmallInts = 16000;   // 64 KB of shared memory

__device__ __forceinline__ void chunk_bounds(const Plan& p, int64_t chunk, int64_t* from, int64_t* to) {
  const int64_t rank = chunk / p.rank_chunks, part = chunk % p.rank_chunks;
  const int64_t end = min((rank + 1) * p.per_rank, p.tokens);
  *from = min(rank * p.per_rank + part * p.chunk_tokens, end);
  *to = min(*from + p.chunk_tokens, end);
}

// A quotient of numbers below 2^22 and 2^11 as a product: 1/size is off by
// 2^-24 relative, the product by less than half a step.
__device__ __forceinline__ int quotient(int e, float inverse) { return (int)((e + 0.5f) * inverse); }

// Counts one token's rows per destination rank.
__device__ __forceinline__ void count_token(const Plan& p, const int32_t* row, float per_size, int* per_rank) {
  uint64_t seen = 0;   // destinations so far, where 64 bits hold them
  for (int j = 0; j < p.top_k; ++j) {
    const int e = row[j];
    if (e < 0 || e >= p.experts) continue;
    const int to = quotient(e, per_size);
    bool counts = true;
    if (p.once && p.ranks <= 64) {
      counts = !(seen >> to & 1);
      seen |= 1ull << to;
    } else if (p.once) {
      for (int h = 0; h < j; ++h)
        counts &= row[h] < 0 || row[h] >= p.experts || quotient(row[h], per_size) != to;
    }
    if (counts) atomicAdd(&per_rank[to], 1);
  }
}

// The places of 64 choices (e < 0: none) of fewer than 2^BITS experts, each
// behind the wave's earlier ones of its expert: next[e] is the expert's next
// place and moves on.  Lanes of the same expert agree in every bit; with the
// number of bits known the ballots overlap (a loop over them took twice as
// long).
template <int BITS>
__device__ __forceinline__ int place_wave(int e, int lane, int* next) {
  const uint64_t some = __ballot(e >= 0);
  uint32_t low = (uint32_t)some, high = (uint32_t)(some >> 32);
#pragma unroll
  for (int bit = 0; bit < BITS; ++bit) {
    const int mine = __builtin_amdgcn_sbfe(e, bit, 1);   // 0 or -1
    const uint64_t set = __ballot(mine != 0);
    low &= ~((uint32_t)set ^ (uint32_t)mine);
    high &= ~((uint32_t)(set >> 32) ^ (uint32_t)mine);
  }
  const int before = (int)__builtin_amdgcn_mbcnt_hi(high, __builtin_amdgcn_mbcnt_lo(low, 0));
  const int all = __popc(low) + __popc(high);
  int place = -1;
  if (e >= 0) place = next[e] + before;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (e >= 0 && before + 1 == all) next[e] = place + 1;  // the last lane of its expert
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return place;
}

// The sum over this lane and the lanes before it.
__device__ __forceinline__ int sum_before(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // 1, 2, 4, 8 lanes on, inside 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // the last lane of the 16 before
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // lane 31
  return v;
}

// The choices of a chunk, 64 at a time: all loads are on their way before
// the first is used.
constexpr int kChunk = 1024;
struct Chunk {
  int64_t from;             // first token
  int n;                    // choices
  int e[kChunk / 64];       // this lane's: choice 64 i + lane; -1 for none
};
__device__ __forceinline__ void load_chunk(const Plan& p, const int32_t* experts, int lane, Chunk* c) {
  int64_t to;
  chunk_bounds(p, blockIdx.x, &c->from, &to);
  c->n = (int)(to - c->from) * p.top_k;
  const int32_t* mine = experts + c->from * p.top_k;
#pragma unroll
  for (int i = 0; i < kChunk / 64; ++i) c->e[i] = i * 64 + lane < c->n ? mine[i * 64 + lane] : -1;
#pragma unroll
  for (int i = 0; i < kChunk / 64; ++i)
    if (c->e[i] < 0 || c->e[i] >= p.experts) c->e[i] = -1;
}

__global__ __launch_bounds__(64) void dispatch_count_kernel(Plan p, const int32_t* __restrict__ experts,
                                                            int32_t* __restrict__ counts, int32_t* __restrict__ sent) {
  extern __shared__ int ints[];
  int* per_expert = ints;
  int* per_rank = per_expert + p.experts;
  int* row = per_rank + p.ranks;       // the chunk's choices
  const int lane = threadIdx.x;
  Chunk c;
  load_chunk(p, experts, lane, &c);
  for (int i = lane; i < p.experts + p.ranks; i += 64) ints[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kChunk / 64; ++i) {
    if (i * 64 >= c.n) break;
    if (c.e[i] >= 0) atomicAdd(&per_expert[c.e[i]], 1);
    row[i * 64 + lane] = c.e[i];
  }
  __syncthreads();
  for (int e = lane; e < p.experts; e += 64) counts[(int64_t)blockIdx.x * p.experts + e] = per_expert[e];
  if (!sent) return;
  const float per_size = 1.0f / (p.experts / p.ranks);
  const int tokens = c.n / p.top_k;
  for (int t = lane; t < tokens; t += 64) count_token(p, row + t * p.top_k, per_size, per_rank);
  __syncthreads();
  for (int d = lane; d < p.ranks; d += 64) sent[(int64_t)blockIdx.x * p.ranks + d] = per_rank[d];
}

// counts[chunk][e] becomes the sum over the chunks before: a workgroup takes
// 16 experts, 64 threads each for as many runs of chunks.  Further
// workgroups add up the traffic, 1,024 pairs of ranks each.
constexpr int kScanExperts = 16, kScanAhead = 16;
__global__ __launch_bounds__(1024) void dispatch_scan_kernel(Plan p, int32_t* __restrict__ counts,
                                                             int32_t* __restrict__ totals,
                                                             const int32_t* __restrict__ sent, double row_bytes,
                                                             double* __restrict__ traffic) {
  const int groups = (p.experts + kScanExperts - 1) / kScanExperts, tid = threadIdx.x;
  if ((int)blockIdx.x >= groups) {
    const int pair = ((int)blockIdx.x - groups) * 1024 + tid;
    if (pair >= p.ranks * p.ranks) return;
    const int from = pair / p.ranks, to = pair % p.ranks;
    int64_t rows = 0;
    const int64_t mine = min(p.rank_chunks, p.chunks - from * p.rank_chunks);   // none or below: no tokens
#pragma unroll 8
    for (int64_t c = 0; c < mine; ++c) rows += sent[(from * p.rank_chunks + c) * p.ranks + to];
    traffic[pair] = (double)rows * row_bytes;
    return;
  }
  __shared__ int runs[64][kScanExperts + 1];
  const int e = blockIdx.x * kScanExperts + tid % kScanExperts, run = tid / kScanExperts;
  const int64_t each = (p.chunks + 63) / 64, first = min(run * each, p.chunks), last = min(first + each, p.chunks);
  // the run's first counts stay in registers, which is all of them up to
  // 1,024 chunks
  int ahead[kScanAhead], sum = 0;
#pragma unroll
  for (int i = 0; i < kScanAhead; ++i) ahead[i] = e < p.experts && first + i < last ? counts[(first + i) * p.experts + e] : 0;
#pragma unroll
  for (int i = 0; i < kScanAhead; ++i) sum += ahead[i];
  if (e < p.experts)
    for (int64_t c = first + kScanAhead; c < last; ++c) sum += counts[c * p.experts + e];
  runs[run][tid % kScanExperts] = sum;
  __syncthreads();
  // a wave per expert over its 64 runs
  const int lane = tid & 63, of = tid >> 6;
  const int mine = runs[lane][of], upto = sum_before(mine);
  __syncthreads();
  runs[lane][of] = upto - mine;
  if (lane == 63 && blockIdx.x * kScanExperts + of < p.experts) totals[blockIdx.x * kScanExperts + of] = upto;
  __syncthreads();
  if (e >= p.experts) return;
  sum = runs[run][tid % kScanExperts];
#pragma unroll
  for (int i = 0; i < kScanAhead; ++i) {
    if (first + i < last) counts[(first + i) * p.experts + e] = sum;
    sum += ahead[i];
  }
  for (int64_t c = first + kScanAhead; c < last; ++c) {
    const int here = counts[c * p.experts + e];
    counts[c * p.experts + e] = sum;
    sum += here;
  }
}

template <int BITS>
__global__ __launch_bounds__(64) void dispatch_place_kernel(Plan p, const int32_t* __restrict__ experts,
                                                            const int32_t* __restrict__ counts,
                                                            const int32_t* __restrict__ totals,
                                                            int32_t* __restrict__ offsets,
                                                            int32_t* __restrict__ token_of_slot,
                                                            int32_t* __restrict__ slot_of_choice) {
  extern __shared__ int next[];  // the next free slot of every expert
  const int lane = threadIdx.x;
  Chunk c;
  load_chunk(p, experts, lane, &c);
  int carry = 0;
  for (int e0 = 0; e0 < p.experts; e0 += 256) {
    int all[4], before[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = e0 + i * 64 + lane;
      all[i] = e < p.experts ? totals[e] : 0;
      before[i] = e < p.experts ? counts[(int64_t)blockIdx.x * p.experts + e] : 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = e0 + i * 64 + lane, upto = sum_before(all[i]);
      if (e < p.experts) {
        const int first = carry + upto - all[i];
        next[e] = first + before[i];
        if (blockIdx.x == 0) offsets[e] = first;
      }
      carry += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  if (blockIdx.x == 0 && lane == 0) offsets[p.experts] = carry;
  // slots that no choice fills
  for (int64_t s = carry + (int64_t)blockIdx.x * 64 + lane; s < p.tokens * p.top_k; s += (int64_t)gridDim.x * 64)
    token_of_slot[s] = -1;
  __syncthreads();
  const float per_token = 1.0f / p.top_k;
#pragma unroll
  for (int i = 0; i < kChunk / 64; ++i) {
    const int at = i * 64 + lane;
    if (i * 64 >= c.n) break;
    const int slot = place_wave<BITS>(c.e[i], lane, next);
    if (slot >= 0) token_of_slot[slot] = (int32_t)c.from + quotient(at, per_token);
    if (at < c.n) slot_of_choice[c.from * p.top_k + at] = slot;
  }
}

// All of it in one workgroup: at most kSmallChoices choices, a sixteenth of
// them per wave, and a traffic matrix that shared memory holds.
template <int BITS>
__global__ __launch_bounds__(1024) void dispatch_small_kernel(Plan p, const int32_t* __restrict__ experts,
                                                              int32_t* __restrict__ offsets,
                                                              int32_t* __restrict__ token_of_slot,
                                                              int32_t* __restrict__ slot_of_choice, double row_bytes,
                                                              double* __restrict__ traffic) {
  extern __shared__ int ints[];
  __shared__ int ends[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = p.experts, pairs = traffic ? p.ranks * p.ranks : 0;
  int* counts = ints;              // [16][E]
  int* sent = ints + 16 * E;       // [ranks][ranks]
  for (int i = tid; i < 16 * E + pairs; i += 1024) ints[i] = 0;
  __syncthreads();
  const int n = (int)p.tokens * p.top_k, each = (n + 1023) / 1024 * 64;   // choices of a wave
  const float per_token = 1.0f / p.top_k, per_size = 1.0f / (E / p.ranks);
  int mine[kSmallChoices / 1024];
#pragma unroll
  for (int h = 0; h < kSmallChoices / 1024; ++h) {
    const int i = wave * each + h * 64 + lane;
    int e = h * 64 < each && i < n ? experts[i] : -1;
    if (e >= E) e = -1;
    mine[h] = e;
    if (e >= 0) atomicAdd(&counts[wave * E + e], 1);
  }
  if (traffic)
    for (int t = tid; t < p.tokens; t += 1024)
      count_token(p, experts + (int64_t)t * p.top_k, per_size, sent + t / (int)p.per_rank * p.ranks);
  __syncthreads();
  // counts to first places: over the waves, then over the experts
  int sum = 0;
  if (tid < E)
    for (int w = 0; w < 16; ++w) {
      const int here = counts[w * E + tid];
      counts[w * E + tid] = sum;
      sum += here;
    }
  const int upto = sum_before(sum);
  if (lane == 63) ends[wave] = upto;
  __syncthreads();
  int first = upto - sum, all = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) first += ends[w];
    all += ends[w];
  }
  if (tid < E) {
    for (int w = 0; w < 16; ++w) counts[w * E + tid] += first;
    offsets[tid] = first;
  }
  if (tid == 0) offsets[E] = all;
  for (int s = all + tid; s < n; s += 1024) token_of_slot[s] = -1;
  for (int i = tid; i < pairs; i += 1024) traffic[i] = (double)sent[i] * row_bytes;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < kSmallChoices / 1024; ++h) {
    if (h * 64 >= each) break;
    const int i = wave * each + h * 64 + lane;
    const int slot = place_wave<BITS>(mine[h], lane, counts + wave * E);
    if (slot >= 0) token_of_slot[slot] = quotient(i, per_token);
    if (i < n) slot_of_choice[i] = slot;
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
  p.chunk_tokens = kChunk / top_k;
  p.rank_chunks = ceil_div(p.per_rank, p.chunk_tokens);
  const int64_t whole = (tokens - 1) / p.per_rank;   // ranks before the last that holds tokens
  p.chunks = whole * p.rank_chunks + ceil_div(tokens - whole * p.per_rank, p.chunk_tokens);
  p.small = tokens * top_k <= kSmallChoices && 16 * experts + ranks * ranks <= kSmallInts;
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
      with_type(type, [&](auto t) {
        with_shape(tokens, r.experts, [&](auto l, auto n) {
          using T = decltype(t);
          constexpr int L = decltype(l)::value, N = decltype(n)::value;
          const size_t lds = r.groups > 1 ? 256 / L * sizeof(float) * (L * N + 1 + 2 * r.groups) : 0;
          const T* in = static_cast<const T*>(d_logits);
          const bool wide = whole_vectors<T>(in, ld_logits, r.experts, Row<T, L, N>::V);
          auto run = [&](auto kernel) {
            in_launches(tokens, kRowsOfLaunch, [&](int64_t first, int64_t rows) {
              hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(rows, 256 / L)), dim3(256), lds,
                                 static_cast<hipStream_t>(hip_stream), r, rows, in + first * ld_logits, ld_logits, wide,
                                 d_bias, d_experts + first * r.top_k, d_weights + first * r.top_k);
            });
          };
          // without a bias and sums of scores the logits give the same order
          const bool by_score = d_bias || r.best > 1;
          if (r.top_k <= 8)
            run(by_score ? route_kernel<T, L, N, true, true> : route_kernel<T, L, N, true, false>);
          else
            run(by_score ? route_kernel<T, L, N, false, true> : route_kernel<T, L, N, false, false>);
        });
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
        hipStream_t s = static_cast<hipStream_t>(hip_stream);
        const T* in = static_cast<const T*>(d_logits);
        T* out = static_cast<T*>(d_dlogits);
        if (r.softmax && !r.renorm) {
          with_shape(tokens, r.experts, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, N = decltype(n)::value, V = Row<T, L, N>::V;
            const bool wide = whole_vectors<T>(in, ld_logits, r.experts, V);
            const bool wide_out = whole_vectors<T>(out, ld_dlogits, r.experts, V);
            in_launches(tokens, kRowsOfLaunch, [&](int64_t first, int64_t rows) {
              hipLaunchKernelGGL((route_back_kernel<T, L, N>), dim3((unsigned)ceil_div(rows, 256 / L)), dim3(256), 0, s, r,
                                 rows, in + first * ld_logits, ld_logits, wide, d_experts + first * r.top_k,
                                 d_dweights + first * r.top_k, out + first * ld_dlogits, ld_dlogits, wide_out);
            });
          });
          return;
        }
        auto run = [&](auto lanes) {
          constexpr int K = decltype(lanes)::value, V = 16 / sizeof(T);
          const size_t lds = 256 / K * sizeof(float) * (ceil_div(r.experts, V) * V);
          const bool wide = whole_vectors<T>(out, ld_dlogits, r.experts, V);
          in_launches(tokens, kRowsOfLaunch, [&](int64_t first, int64_t rows) {
            hipLaunchKernelGGL((route_back_chosen_kernel<T, K>), dim3((unsigned)ceil_div(rows, 256 / K)), dim3(256), lds, s,
                               r, rows, in + first * ld_logits, ld_logits, d_experts + first * r.top_k,
                               d_dweights + first * r.top_k, out + first * ld_dlogits, ld_dlogits, wide);
          });
        };
        // the rows of a workgroup have to fit its shared memory (64 KB)
        if (r.top_k <= 8 && r.experts <= 512)
          run(std::integral_constant<int, 8>{});
        else if (r.top_k <= 16)
          run(std::integral_constant<int, 16>{});
        else
          run(std::integral_constant<int, 32>{});
      });
    });
  });
}

extern "C" int64_t netsim_dispatch_work_bytes(int32_t experts, int32_t top_k, int64_t tokens, int32_t ranks,
                                              int64_t tokens_per_rank) {
  if (bad_dispatch(experts, top_k, tokens, ranks, tokens_per_rank)) return -1;
  if (tokens == 0) return 0;
  const Plan p = make_plan(experts, top_k, tokens, ranks, tokens_per_rank, false);
  // one workgroup works in its own memory: a word, so that there is an array
  return p.small ? 4 : 4 * (p.chunks * (p.experts + p.ranks) + p.experts);
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
      if (p.small) {
        auto run = [&](auto kernel) {
          hipLaunchKernelGGL(kernel, dim3(1), dim3(1024), sizeof(int) * (16 * experts + (d_traffic ? ranks * ranks : 0)),
                             s, p, d_experts, d_offsets, d_token_of_slot, d_slot_of_choice, row_bytes, d_traffic);
        };
        run(experts <= 64 ? dispatch_small_kernel<6> : experts <= 256 ? dispatch_small_kernel<8> : dispatch_small_kernel<10>);
        return;
      }
      int32_t* counts = static_cast<int32_t*>(d_work);
      int32_t* sent = counts + p.chunks * p.experts;
      int32_t* totals = sent + p.chunks * p.ranks;
      hipLaunchKernelGGL(dispatch_count_kernel, dim3((unsigned)p.chunks), dim3(64),
                         sizeof(int) * (experts + ranks + kChunk), s, p, d_experts, counts, d_traffic ? sent : nullptr);
      const int64_t scans = ceil_div(experts, kScanExperts) + (d_traffic ? ceil_div((int64_t)ranks * ranks, 1024) : 0);
      hipLaunchKernelGGL(dispatch_scan_kernel, dim3((unsigned)scans), dim3(1024), 0, s, p, counts, totals, sent,
                         row_bytes, d_traffic);
      auto place = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)p.chunks), dim3(64), sizeof(int) * experts, s, p, d_experts, counts,
                           totals, d_offsets, d_token_of_slot, d_slot_of_choice);
      };
      place(experts <= 64 ? dispatch_place_kernel<6> : experts <= 256 ? dispatch_place_kernel<8> : dispatch_place_kernel<10>);
    });
  });
}
