// Matrix products by tiles: what the products of experts (experts.hip) and
// those in 8 bits (eight.hip) share.
//
// A workgroup computes a tile of BM rows and BN columns.  A step brings 128
// bytes of the summed index of both operands into shared memory; two stages
// alternate, so the next step's loads are in flight while the matrix cores
// work on this one.  An operand lies in memory with the summed index as its
// fast one (RowTile) or as its slow one (ColTile, 16-bit values only); it goes
// to shared memory as it lies, in chunks of 16 bytes whose place is exclusive-
// ored with the row, so that neither the stores nor the matrix cores' reads
// meet in a bank: a read of 16 lanes takes one chunk each of 16 rows, a
// transposing one 64 bytes each of four.
#pragma once

#include "values.h"

namespace netsim_ops {
namespace {

constexpr int kStepBytes = 128;
using i32x4 = __attribute__((ext_vector_type(4))) int;
using i32x16 = __attribute__((ext_vector_type(16))) int;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;

// What a chunk outside its array is read from.
__device__ const uint4 zeros = {0, 0, 0, 0};

// Products of 32 x 32 over 32 bytes of the summed index; a lane gives 16 bytes
// of row (lane & 31) from byte 16 (lane >> 5) on, and gets of column
// (lane & 31) the rows 8 (r >> 2) + 4 (lane >> 5) + (r & 3).
template <class T>
struct Matrix;
template <>
struct Matrix<bf16> {
  using Sum = f32x16;
  static __device__ __forceinline__ Sum add(uint4 a, uint4 b, Sum c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Matrix<f16> {
  using Sum = f32x16;
  static __device__ __forceinline__ Sum add(uint4 a, uint4 b, Sum c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Matrix<int8_t> {
  using Sum = i32x16;
  static __device__ __forceinline__ Sum add(uint4 a, uint4 b, Sum c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// 16 bytes of every lane to consecutive places of shared memory from address
// `to` on (the same for the wave), without passing through registers.  Written
// out, as the compiler would wait for such loads before any read of shared
// memory; the wait is in Tile::run, before the barrier that hands the stage over.
__device__ __forceinline__ void to_shared(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "memory");
}

__device__ __forceinline__ int wave_of_group() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// A place in shared memory, and its address there.
struct Place {
  char* at;
  uint32_t address;
  __device__ __forceinline__ Place operator+(int n) const { return {at + n, address + n}; }
};
__device__ __forceinline__ Place place_of(char* shared) {
  const uint32_t address = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)shared;
  return {shared, (uint32_t)__builtin_amdgcn_readfirstlane(address)};
}

// A chunk of 16 bytes of which `left` elements are there, zeros beyond.
template <class T>
__device__ __forceinline__ uint4 chunk_of(const T* p, int left) {
  const Eight<T> v = load_some(p, left);
  return make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
}

// Rows of which a step takes 128 bytes each.  DIRECT: rows start at multiples
// of 16 bytes and have whole chunks.
template <class T, int R, int THREADS, bool DIRECT>
struct RowTile {
  static constexpr int N = R * 8 / THREADS, PER = 16 / sizeof(T), STEP = kStepBytes / sizeof(T);
  static_assert(THREADS / 8 % 16 == 0 && N * THREADS == R * 8, "a thread's chunks have the same place in their rows");
  const T* at[N];
  uint4 held[DIRECT ? 1 : N];
  int col;

  // row(r): where row r of the tile starts (a row that may be read).
  template <class F>
  __device__ __forceinline__ void open(F&& row) {
    const int r = threadIdx.x >> 3;
    col = ((threadIdx.x & 7) ^ ((r >> 1) & 7)) * PER;
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = row(r + i * (THREADS / 8)) + col;
  }
  // Step from element k0 of rows of k elements; shift: of another array of
  // such rows.
  __device__ __forceinline__ void load(Place stage, int k0, int k, int64_t shift = 0) {
    const int left = k - k0 - col, wave = wave_of_group();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const T* from = at[i] + shift + k0;
      if constexpr (DIRECT)
        to_shared(left > 0 ? static_cast<const void*>(from) : &zeros, stage.address + i * THREADS * 16 + wave * 1024);
      else
        held[i] = chunk_of(from, left);
    }
  }
  __device__ __forceinline__ void store(Place stage) {
    if constexpr (!DIRECT)
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(stage.at + (i * THREADS + threadIdx.x) * 16) = held[i];
  }
  // The operand of rows first .. first + 31, bytes 32 h .. of the step.
  static __device__ __forceinline__ uint4 operand(const char* stage, int first, int h) {
    const int lane = threadIdx.x & 63;
    return *reinterpret_cast<const uint4*>(stage + (first + (lane & 31)) * kStepBytes +
                                           ((((lane >> 5) ^ (lane >> 1)) & 7) * 16 ^ 32 * h));
  }
};

// The summed index as the slow one: 64 rows of R columns each.
template <class T, int R, int THREADS, bool DIRECT>
struct ColTile {
  static_assert(sizeof(T) == 2 && R >= 128, "");
  static constexpr int CHUNKS = R / 8, N = R * 8 / THREADS, EACH = THREADS / CHUNKS, STEP = 64;
  static_assert(EACH % 4 == 0 && EACH * N == STEP, "a thread's chunks have the same place in their rows");
  const T* at;
  int64_t ld;
  uint4 held[DIRECT ? 1 : N];
  int left;

  __device__ __forceinline__ int row(int i) const { return threadIdx.x / CHUNKS + i * EACH; }
  __device__ __forceinline__ void open(const T* base, int64_t pitch, int c0, int cols) {
    const int c = c0 + (threadIdx.x % CHUNKS ^ (4 * (row(0) & 3))) * 8;
    left = cols - c;
    at = base + c;
    ld = pitch;
  }
  // Rows r(i) of the array, i: this thread's chunks; none where r is negative.
  template <class F>
  __device__ __forceinline__ void load(Place stage, F&& r, int64_t shift = 0) {
    const int wave = wave_of_group();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t n = r(i);
      const T* from = at + shift + n * ld;
      if constexpr (DIRECT)
        to_shared(left > 0 && n >= 0 ? static_cast<const void*>(from) : &zeros, stage.address + i * THREADS * 16 + wave * 1024);
      else
        held[i] = chunk_of(from, n >= 0 ? left : 0);
    }
  }
  __device__ __forceinline__ void store(Place stage) {
    if constexpr (!DIRECT)
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(stage.at + (i * THREADS + threadIdx.x) * 16) = held[i];
  }
  // Lanes 0-15 give four rows of 16 columns and get a column each; lanes 16-31
  // the next 16 columns, lanes 32-63 the rows 8 further on.
  static __device__ __forceinline__ uint4 operand(const char* stage, int first, int h) {
    const int lane = threadIdx.x & 63, k = (lane >> 5) * 8 + ((lane >> 2) & 3);
    const int chunk = (first / 8 ^ (4 * (k & 3))) + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    const char* from = stage + (h * 16 + k) * R * 2 + chunk * 16 + (lane & 1) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 4 * R * 2));
    return __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// A tile's sums and where a wave's part of them lies: WM x WN waves, each with
// FM x FN products of 32 x 32.
template <class T, int BM, int BN, int WM, int WN>
struct Tile {
  static constexpr int THREADS = 64 * WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
  static constexpr int STAGE = (BM + BN) * kStepBytes, LDS = 2 * STAGE;
  using M = Matrix<T>;
  typename M::Sum sum[FM][FN];

  __device__ __forceinline__ Tile() {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) sum[i][j] = typename M::Sum{};
  }
  static __device__ __forceinline__ int row0() { return wave_of_group() / WN * (BM / WM); }
  static __device__ __forceinline__ int col0() { return wave_of_group() % WN * (BN / WN); }

  // `count` steps; load(stage, s) brings in step s, store(stage) what of it
  // went to registers.  At the end no wave reads shared memory any more.
  template <class A, class B, class Load, class Store>
  __device__ __forceinline__ void run(char* shared, int count, Load&& load, Store&& store) {
    if (count <= 0) return;
    const Place first = place_of(shared), second = first + STAGE;
    const int a0 = row0(), b0 = col0();
    load(first, 0);
    store(first);
    auto hand_over = [] {   // what the next step reads is in shared memory, for every wave
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    };
    auto step = [&](int s, Place stage, Place next) {
      const bool more = s + 1 < count;
      if (more) load(next, s + 1);
      // the next operands are read while the matrix cores work on these
      uint4 a[2][FM], b[2][FN];
      auto operands = [&](int h) {
#pragma unroll
        for (int j = 0; j < FN; ++j) b[h & 1][j] = B::operand(stage.at + BM * kStepBytes, b0 + j * 32, h);
#pragma unroll
        for (int i = 0; i < FM; ++i) a[h & 1][i] = A::operand(stage.at, a0 + i * 32, h);
      };
      operands(0);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        if (h < 3) operands(h + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) sum[i][j] = M::add(b[h & 1][j], a[h & 1][i], sum[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (more) store(next);
      hand_over();
    };
    hand_over();
    int s = 0;
    for (; s + 1 < count; s += 2) {
      step(s, first, second);
      step(s + 1, second, first);
    }
    if (s < count) step(s, first, second);
  }

  // Writes rows 0 .. rows-1 and columns 0 .. cols-1 of the tile to `out`,
  // through shared memory, so that rows leave as whole lines.  value(i, j, r):
  // what comes of the sums; JN fragments of 32 columns a wave, at col(j).
  template <int COLS, int JN, class O, class C, class F>
  static __device__ __forceinline__ void write(char* shared, O* out, int64_t ld, int rows, int cols, C&& col, F&& value) {
    constexpr int V = 16 / sizeof(O), PITCH = COLS + V;
    constexpr int FIT = LDS / (PITCH * (int)sizeof(O));
    constexpr int ROWS = FIT >= BM ? BM : FIT >= BM / 2 ? BM / 2 : BM / 4;   // of a pass
    static_assert(ROWS % 32 == 0 && ROWS <= FIT, "");
    const int lane = threadIdx.x & 63;
    O* tile = reinterpret_cast<O*>(shared);
    const bool wide = ld % V == 0 && cols % V == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
#pragma unroll
    for (int first = 0; first < BM; first += ROWS) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int m = row0() + i * 32 - first;
        if (m < 0 || m >= ROWS) continue;   // the same for a wave
#pragma unroll
        for (int j = 0; j < JN; ++j)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            struct alignas(4 * sizeof(O)) Four {
              O v[4];
            } four;
#pragma unroll
            for (int h = 0; h < 4; ++h) four.v[h] = (O)value(i, j, r + h);
            *reinterpret_cast<Four*>(tile + (m + (lane & 31)) * PITCH + col(j) + r * 2 + (lane >> 5) * 4) = four;
          }
      }
      __syncthreads();
      if (wide) {
#pragma unroll 4
        for (int t = threadIdx.x; t < ROWS * COLS / V; t += THREADS) {
          const int m = t / (COLS / V), c = t % (COLS / V) * V;
          if (first + m < rows && c < cols)
            *reinterpret_cast<uint4*>(out + (first + m) * ld + c) = *reinterpret_cast<const uint4*>(tile + m * PITCH + c);
        }
      } else {
#pragma unroll 4
        for (int t = threadIdx.x; t < ROWS * COLS; t += THREADS) {
          const int m = t / COLS, c = t % COLS;
          if (first + m < rows && c < cols) out[(first + m) * ld + c] = tile[m * PITCH + c];
        }
      }
    }
  }
};

// ------------------------------------------------------- rows of experts
// Slots from .. to-1 of an expert; expert -1: slots of no expert, -2: none.
struct Rows {
  int expert, from, to;
};

// Inclusive sums over the lanes of a wave.
__device__ __forceinline__ int lanes_up(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);    // 1 lane down a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);    // 2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);    // 4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);    // 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // lane 15 of the row before, rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // lane 31, rows 2 and 3
  return v;
}

// Tile number `want` when every expert's slots are cut into tiles of `size`:
// the experts' slots, then those before the first one's and those behind the
// last one's.  offsets NULL: one expert has all slots.
__device__ __forceinline__ Rows find_rows(const int32_t* offsets, int experts, int slots, int size, int want) {
  auto part = [&](int expert, int from, int to, int nth) {
    const int64_t start = from + (int64_t)nth * size;
    return start < to ? Rows{expert, (int)start, (int)min(start + size, (int64_t)to)} : Rows{-2, 0, 0};
  };
  if (!offsets) return part(0, 0, slots, want);
  const int lane = threadIdx.x & 63;
  for (int first = 0; first < experts; first += 64) {
    const int e = first + lane;
    int a = 0, b = 0;
    if (e < experts) {
      a = min(max(offsets[e], 0), slots);
      b = min(max(offsets[e + 1], a), slots);
    }
    const int tiles = (int)(((int64_t)b - a + size - 1) / size), up = lanes_up(tiles);
    const uint64_t found = __ballot(want >= up - tiles && want < up);
    if (found) {
      const int at = __builtin_ctzll(found);
      return part(first + at, __builtin_amdgcn_readlane(a, at), __builtin_amdgcn_readlane(b, at),
                  want - __builtin_amdgcn_readlane(up - tiles, at));
    }
    want -= __builtin_amdgcn_readlane(up, 63);
  }
  const int head = min(max(offsets[0], 0), slots), tail = min(max(offsets[experts], 0), slots);
  const int tiles = (int)(((int64_t)head + size - 1) / size);
  return want < tiles ? part(-1, 0, head, want) : part(-1, tail, slots, want - tiles);
}

// How many such tiles there may be.
inline int64_t most_rows_tiles(int64_t experts, int64_t slots, int64_t size, bool offsets) {
  if (!offsets) return ceil_div(slots, size);
  return slots / size + (experts + 2 < slots ? experts + 2 : slots);
}

// Workgroups go to the 8 dies in turn: tiles are numbered so that 32
// consecutive ones, which share rows and columns, meet in one die's cache.
constexpr int kDies = 8, kNear = 32;
__device__ __forceinline__ int64_t tile_of_group(uint32_t group) {
  const uint32_t die = group % kDies, nth = group / kDies;
  return ((int64_t)(nth / kNear) * kDies + die) * kNear + nth % kNear;
}
constexpr int64_t kMaxGroups = 1 << 22;   // of a launch: at most 2^31 threads, whole rounds of dies

// Launches that together have a workgroup for each of `tiles` tiles: go(first,
// groups), for groups numbered by tile_of_group from `first` on.
template <class F>
void over_tiles(int64_t tiles, F&& go) {
  const int64_t groups = ceil_div(tiles, kDies * kNear) * kDies * kNear;
  in_launches(groups, kMaxGroups, [&](int64_t first, int64_t n) { go(first, (unsigned)n); });
}

}  // namespace
}  // namespace netsim_ops
