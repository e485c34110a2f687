// Sums over the slots of experts: how a call's are cut into parts, so that
// all compute units have work to the end however uneven the experts are, and
// how the parts are joined (act.hip, experts.hip).
#pragma once

#include "ops.h"

namespace netsim_ops {
namespace {

constexpr int kMaxCols = 1 << 20;
constexpr int64_t kMaxSlots = 0x7fffffff - 4096;   // a step past the end stays in 32 bits

// experts matrices [n x cols], each a sum over the expert's slots.
struct Sums {
  int experts, n, cols, slots;
  bool wide_joins;   // four elements of dW at a time are aligned
};

// A part of an expert's slots.  partial < 0: the whole sum, written to dW;
// otherwise the number of the partial sum in the workspace.
struct alignas(16) Item {
  int expert, from, to, partial;
};

// An expert whose sum is in parts: `parts` partial sums from `first` on.
struct alignas(16) Join {
  int expert, first, parts, unused;
};

// The bounds of an expert's slots, held to the arrays; offsets NULL: all slots.
__device__ __forceinline__ Item segment(const int32_t* offsets, int e, int slots) {
  if (!offsets) return Item{e, 0, slots, -1};
  const int a = min(max(offsets[e], 0), slots), b = min(max(offsets[e + 1], a), slots);
  return Item{e, a, b, -1};
}

// How the sums of a call are cut.  An expert with more than `longest` slots
// is cut into equal parts of at most that many.
struct Cut {
  int tile;          // rows and columns of dW a workgroup computes
  int step;          // slots of one pass through shared memory
  int64_t longest;
  int64_t items, partials, joins;   // at most
  // Who lays out the parts: no one (whole sums, in the experts' order), every
  // wave that needs one by itself, or plan_kernel in a list.
  enum Plan { WHOLE, BY_WAVE, LISTED } plan;
  int64_t bytes;     // workspace
};

// The parts of an expert's sum, and the slots of each.
__device__ __forceinline__ void cut_sum(const Cut& cut, uint32_t n, uint32_t* parts, uint32_t* each) {
  const uint32_t longest = (uint32_t)cut.longest;
  *parts = n > longest ? (n + longest - 1) / longest : 1;
  *each = ((n + *parts - 1) / *parts + cut.step - 1) / cut.step * cut.step;
  if (*parts > 1) *parts = (n + *each - 1) / *each;
}

// Part number `want` (JOINS: the want-th expert that is cut) in the order of
// plan_kernel, by a wave, a lane per expert: for few experts less than the
// launch that would write a list.
template <bool JOINS>
__device__ __forceinline__ void find_part(const Sums& g, const Cut& cut, const int32_t* offsets, int want, Item* part,
                                          Join* joined) {
  const int e = threadIdx.x & 63;
  Item it{-1, 0, 0, -1};
  uint32_t parts = 0, each = 0;
  if (e < g.experts) {
    it = segment(offsets, e, g.slots);
    cut_sum(cut, (uint32_t)(it.to - it.from), &parts, &each);
  }
  int item = 0, partial = 0, join = 0;
  for (int h = 0; h < g.experts; ++h) {
    const int other = __builtin_amdgcn_readlane((int)each, h), count = __builtin_amdgcn_readlane((int)parts, h);
    const bool before = other > (int)each || (other == (int)each && h < e);
    item += before ? count : 0;
    partial += before && count > 1 ? count : 0;
    join += before && count > 1 ? 1 : 0;
  }
  const bool fits = item + (int64_t)parts <= cut.items && (parts == 1 || partial + (int64_t)parts <= cut.partials);
  const uint64_t found = __ballot(e < g.experts && fits &&
                                  (JOINS ? parts > 1 && join == want : want >= item && want < item + (int)parts));
  const int lane = found ? __builtin_ctzll(found) : 0;
  auto of = [&](int v) { return __builtin_amdgcn_readlane(v, lane); };
  if constexpr (JOINS) {
    const Join all{of(e), of(partial), of((int)parts), 0};
    *joined = found ? all : Join{-1, 0, 0, 0};
  } else {
    const int count = of((int)parts), slots = of((int)each), p = want - of(item), first = of(it.from), last = of(it.to);
    const int64_t from = first + (int64_t)p * slots, to = min((int64_t)last, from + slots);
    const int number = of(partial) + p, expert = of(e);
    *part = !found ? Item{-1, 0, 0, -1} : count > 1 ? Item{expert, (int)from, (int)to, number} : Item{expert, first, last, -1};
  }
}

// Orders the experts' sums by length, longest first, and cuts the long ones:
// workgroups start in this order, so the last to end are short (a sum over
// the hot expert of 131,072 routed slots, 25,480 long, started last would
// add 15%).
// One workgroup with a thread per expert.
__global__ __launch_bounds__(1024) void plan_kernel(Sums g, Cut cut, const int32_t* __restrict__ offsets,
                                                    Item* __restrict__ items, Join* __restrict__ joins) {
  __shared__ int length[1024], first_item[1024], first_partial[1024];
  __shared__ Item whole[1024];     // by place in the order; `partial` holds the slots of a part
  __shared__ int sums[3][16];
  const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
  Item it{-1, 0, 0, 0};
  uint32_t parts = 0, each = 0;
  if (e < g.experts) {
    it = segment(offsets, e, g.slots);
    cut_sum(cut, (uint32_t)(it.to - it.from), &parts, &each);
    it.partial = (int)each;
  }
  length[e] = e < g.experts ? (int)each : -1;
  __syncthreads();
  int place = e;
  if (e < g.experts) {
    place = 0;
#pragma unroll 8
    for (int h = 0; h < g.experts; ++h) place += length[h] > (int)each || (length[h] == (int)each && h < e);
  }
  whole[place] = it;
  first_item[place] = parts;
  __syncthreads();
  // per place: the parts, partial sums and joins of the places before
  const int here = first_item[e], cuts = here > 1 ? here : 0;
  int v[3] = {here, cuts, cuts ? 1 : 0};
#pragma unroll
  for (int i = 0; i < 3; ++i) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int w = __shfl_up(v[i], o, 64);
      if (lane >= o) v[i] += w;
    }
    if (lane == 63) sums[i][wave] = v[i];
  }
  __syncthreads();
  int all_items = 0, all_joins = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    if (w < wave)
      for (int i = 0; i < 3; ++i) v[i] += sums[i][w];
    all_items += sums[0][w];
    all_joins += sums[2][w];
  }
  // offsets that decrease could ask for more than there is room for: such
  // sums are left out
  const int item = v[0] - here, partial = v[1] - cuts, join = v[2] - (cuts ? 1 : 0);
  const bool fits = item + here <= cut.items && partial + cuts <= cut.partials;
  first_item[e] = item;
  first_partial[e] = !fits ? -2 : cuts ? partial : -1;
  if (cuts && join < cut.joins) joins[join] = fits ? Join{whole[e].expert, partial, here, 0} : Join{-1, 0, 0, 0};
  for (int64_t i = all_joins + e; i < cut.joins; i += blockDim.x) joins[i] = Join{-1, 0, 0, 0};
  __syncthreads();
  for (int i = e; i < cut.items; i += blockDim.x) {
    Item out{-1, 0, 0, -1};
    if (i < all_items) {
      int low = 0, high = g.experts;   // the last place whose first item is at most i
      while (high - low > 1) {
        const int mid = (low + high) / 2;
        (first_item[mid] <= i ? low : high) = mid;
      }
      const Item w = whole[low];
      const int p = i - first_item[low], before = first_partial[low];
      const int64_t from = w.from + (int64_t)p * w.partial, to = min((int64_t)w.to, from + w.partial);
      if (before == -1)
        out = Item{w.expert, w.from, w.to, -1};
      else if (before >= 0)
        out = Item{w.expert, (int)from, (int)to, before + p};
    }
    items[i] = out;
  }
}

// dW of the experts whose sums are in parts.  Four threads take every fourth
// part of four elements; the order of the sum depends on the parts alone.
template <class O>
__global__ __launch_bounds__(256) void join_kernel(Sums g, Cut cut, const int32_t* __restrict__ offsets,
                                                   const Join* __restrict__ joins,
                                                   const float* __restrict__ partials, O* __restrict__ dw) {
  __shared__ float sums[4][64][4];
  Join j;
  if (cut.plan == Cut::LISTED)
    j = joins[blockIdx.y];
  else
    find_part<true>(g, cut, offsets, blockIdx.y, nullptr, &j);
  if (j.parts == 0) return;
  const int64_t size = (int64_t)g.n * g.cols;
  const float* from = partials + j.first * size;
  O* out = dw + j.expert * size;
  const int quarter = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int64_t i0 = (int64_t)blockIdx.x * 256; i0 < size; i0 += (int64_t)gridDim.x * 256) {
    const int64_t i = i0 + lane * 4;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g.wide_joins) {
      if (i < size) {
#pragma unroll 4
        for (int p = quarter; p < j.parts; p += 4) {
          const float4 v = *reinterpret_cast<const float4*>(from + p * size + i);
          sum[0] += v.x;
          sum[1] += v.y;
          sum[2] += v.z;
          sum[3] += v.w;
        }
      }
    } else {
      for (int h = 0; h < 4; ++h)
        if (i + h < size)
          for (int p = quarter; p < j.parts; p += 4) sum[h] += from[p * size + i + h];
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) sums[quarter][lane][h] = sum[h];
    __syncthreads();
    if (quarter == 0 && i < size) {
      struct alignas(4 * sizeof(O)) Four {
        O v[4];
      } four;
#pragma unroll
      for (int h = 0; h < 4; ++h)
        four.v[h] = (O)((sums[0][lane][h] + sums[1][lane][h]) + (sums[2][lane][h] + sums[3][lane][h]));
      if (g.wide_joins) {
        *reinterpret_cast<Four*>(out + i) = four;
      } else {
        for (int h = 0; h < 4; ++h)
          if (i + h < size) out[i + h] = four.v[h];
      }
    }
    __syncthreads();
  }
}

}  // namespace
}  // namespace netsim_ops
