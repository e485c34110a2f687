// Activations saved in 8 bits, and the experts' weight gradients from them.
//
// A saved row holds, per block of 32 columns, an exponent e and 32 signed
// whole numbers q with x ~ q 2^e: e = floor(log2 of the largest magnitude)
// - 6, at least -126, and q = x 2^-e rounded to nearest even, held to
// +-127.  The step is a power of two, so q 2^e has at most 7 significant
// bits and is a bfloat16 without rounding: a matrix product reads the saved
// rows exactly, and its only roundings are those of its 32-bit sums.
#include <math.h>

#include "ops.h"
#include "parts.h"
#include "values.h"

namespace netsim_ops {
namespace {

constexpr int kBlock = 32;          // columns that share an exponent
constexpr int kNotFinite = -128;    // exponent of a block that held an infinity or a NaN

// 2^e as a float, -126 <= e <= 127.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// ----------------------------------------------------------- save, restore
// Both pass over the data once and are bound by memory.  A lane takes half a
// block (16 columns: 16 bytes of q, 32 or 64 of x), so a block's largest
// magnitude is one exchange between neighbours away.  32,768 rows of 4,096
// bfloat16 columns: saved in 82 us, restored in 67 us (407 MB each: 4.9 and
// 6.0 TB/s; a large copy reaches 4.9).
struct Unit {
  int64_t row, block;   // row and block, counted over all rows
  int col;
};
// The half block of this thread: number blockIdx.x * 256 + threadIdx.x.
__device__ __forceinline__ Unit unit_of(int blocks) {
  const uint32_t per_row = 2 * blocks;
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / per_row;   // the same for the workgroup
  const uint32_t at = (uint32_t)(first - row0 * per_row) + threadIdx.x, rows = at / per_row;
  return Unit{row0 + rows, (first + threadIdx.x) >> 1, (int)(at - rows * per_row) * 16};
}

template <class T>
__global__ __launch_bounds__(256) void save_kernel(int64_t rows, int cols, int blocks, const T* __restrict__ x,
                                                   int64_t ld, int8_t* __restrict__ q, int8_t* __restrict__ exponents) {
  const Unit u = unit_of(blocks);
  if (u.row >= rows) return;
  const T* from = x + u.row * ld + u.col;
  float v[16], top = 0.0f;
  bool odd = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const Eight<T> in = load_some(from + 8 * h, cols - u.col - 8 * h);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[8 * h + j] = value_of(in, j);
      odd |= !isfinite(v[8 * h + j]);
      top = fmaxf(top, fabsf(v[8 * h + j]));
    }
  }
  top = fmaxf(top, __shfl_xor(top, 1, 64));   // the other half: the next thread, of the same row
  odd |= __shfl_xor((int)odd, 1, 64) != 0;
  int e = (int)(__float_as_uint(top) >> 23) - 127 - 6;
  e = e < -126 ? -126 : e;
  const float up = pow2(-e);
  uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float r = odd ? 0.0f : fminf(fmaxf(rintf(v[j] * up), -127.0f), 127.0f);
    word[j >> 2] |= (uint32_t)(uint8_t)(int8_t)(int)r << (8 * (j & 3));
  }
  *reinterpret_cast<uint4*>(q + u.block * kBlock + (u.col & 16)) = make_uint4(word[0], word[1], word[2], word[3]);
  if ((u.col & 16) == 0) exponents[u.block] = odd ? (int8_t)kNotFinite : (int8_t)e;
}

template <class T>
__global__ __launch_bounds__(256) void restore_kernel(int64_t rows, int cols, int blocks,
                                                      const int8_t* __restrict__ q,
                                                      const int8_t* __restrict__ exponents, T* __restrict__ x,
                                                      int64_t ld) {
  const Unit u = unit_of(blocks);
  if (u.row >= rows) return;
  const int e = exponents[u.block];
  const float step = e == kNotFinite ? NAN : pow2(e);
  const uint4 in = *reinterpret_cast<const uint4*>(q + u.block * kBlock + (u.col & 16));
  const uint32_t word[4] = {in.x, in.y, in.z, in.w};
  T* to = x + u.row * ld + u.col;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(word[2 * h + (j >> 2)] >> (8 * (j & 3))) * step;
    store_some(to + 8 * h, v, cols - u.col - 8 * h);
  }
}

// --------------------------------------------------------- weight gradient
// dW[e][n][c] = sum over the slots s of expert e of dy[s][n] x[row(s)][c].
// The sum runs over slots, so both factors lie with the summed index as
// their slow one: tiles of KB slots go to shared memory as they lie, and the
// matrix cores' operands (eight slots of one column in a lane) come from
// transposing reads.  Saved rows are widened to bfloat16 on their way into
// shared memory, once per workgroup.  dy enters as bfloat16: one term for
// bfloat16, two for float16 and three for float32, whose sum is the value
// without rounding (down to bfloat16's smallest magnitude).
struct Grad : Sums {
  int blocks;
  int64_t rows, ld;
  // -1: a slot's row is map[slot]; 0: the slot itself (map is then any word
  // that may be read).  A mask, so that no branch parts the step's products.
  int mapped;
};

template <class T>
struct Terms {
  static constexpr int value = 3;
};
template <>
struct Terms<bf16> {
  static constexpr int value = 1;
};
template <>
struct Terms<f16> {
  static constexpr int value = 2;
};

// The upper halves of two floats: bfloat16 with what does not fit cut off
// (never an overflow), a in the low half.
__device__ __forceinline__ uint32_t pack(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

template <class T, class O, int BN, int BC, int WN, int WC, int KB>
__global__ __launch_bounds__(64 * WN * WC) void grad_kernel(Grad g, Cut cut, const Item* __restrict__ items,
                                                            const T* __restrict__ dy, const int8_t* __restrict__ q,
                                                            const int8_t* __restrict__ exponents,
                                                            const int32_t* __restrict__ map,
                                                            const int32_t* __restrict__ offsets, O* __restrict__ dw,
                                                            float* __restrict__ partials) {
  constexpr int THREADS = 64 * WN * WC, TERMS = Terms<T>::value;
  // 64 bytes more than a row: the four rows of a transposing read of 32
  // columns lie in different quarters of the banks
  constexpr int PY = BN + 32, PX = BC + 32, STAGE = KB * (TERMS * PY + PX);
  constexpr int CY = BN / 8, NY = KB * CY / THREADS, CX = BC / 16, NX = KB * CX / THREADS;
  constexpr int FN = BN / WN / 32, FC = BC / WC / 32;
  static_assert(THREADS % CY == 0 && THREADS % CX == 0 && NY * THREADS == KB * CY && NX * THREADS == KB * CX, "");
  static_assert(CY == 2 * CX && NY == 2 * NX, "a wave's slots of dy are those of its saved rows");
  constexpr float MOST = sizeof(T) == 2 ? 65504.0f : 3.402823466e38f;
  extern __shared__ __align__(16) bf16 shared[];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_n = (g.n + BN - 1) / BN;
  const int n0 = (int)(blockIdx.x % tiles_n) * BN, c0 = (int)(blockIdx.x / tiles_n) * BC;
  Item it;
  if (cut.plan == Cut::WHOLE)
    it = segment(offsets, blockIdx.y, g.slots);
  else if (cut.plan == Cut::LISTED)
    it = items[blockIdx.y];
  else
    find_part<false>(g, cut, offsets, blockIdx.y, &it, nullptr);
  if (it.expert < 0) return;
  if (g.rows == 0) it.to = it.from;   // no row to read: every slot is left out

  // This thread's part of a tile of dy and of saved rows.  A wave brings in
  // dy of the slots whose saved rows it brings in, half of them at a time.
  const int y_chunk = tid % CY, x_chunk = tid % CX, x_row = tid / CX;
  const int y_row = wave * (64 / CX) + lane / CY;
  auto y_step = [](int i) { return (i & 1) * (64 / CY) + (i >> 1) * (THREADS / CX); };
  const int y_left = g.n - (n0 + y_chunk * 8);
  const bool x_in = c0 + x_chunk * 16 < g.blocks * kBlock;
  // columns beyond the row reach no output: a chunk wholly beyond reads the
  // row's first one
  const T* y_at = dy + (int64_t)(it.from + y_row) * g.ld + (y_left > 0 ? n0 + y_chunk * 8 : 0);
  const int64_t x_at = x_in ? (int64_t)(c0 + x_chunk * 16) / kBlock : 0;
  // Tiles wholly inside the part are read without conditions; a row's last
  // chunk then reads into the next row, so not where there is none.
  const int plain_to = it.to - (it.to == g.slots && g.n % 8 != 0);
  const bool y_wide = g.n >= 8;
  const uint32_t row_limit = (uint32_t)min(g.rows, (int64_t)0x80000000);
  Eight<T> y[NY];
  uint4 x[NX];
  int row[NX];
  uint8_t e[NX];   // as loaded: widening it would wait for it
  bool held[NX];   // whether x and e are a row's
  uint64_t stored[NX];   // the lanes whose held was set when their x was stored

  auto load_rows = [&](int s0) {
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int s = s0 + x_row + i * (THREADS / CX);
      row[i] = map[min(s, it.to - 1) & g.mapped];   // not looked at before the next step
    }
  };
  auto load_y = [&](int s0, int i, bool plain) {
    const T* from = y_at + (int64_t)(s0 - it.from + y_step(i)) * g.ld;
    if (plain)
      y[i] = load_eight(from);
    else
      y[i] = load_some(from, s0 + y_row + y_step(i) < it.to ? y_left : 0);
  };
  auto load_x = [&](int s0, int i) {
    // no conditions that branch: the products on both sides stay one block
    const int s = s0 + x_row + i * (THREADS / CX), r = (row[i] & g.mapped) | (s & ~g.mapped);
    held[i] = (s < it.to) & ((uint32_t)r < row_limit);
    const int64_t block = (int64_t)(held[i] ? r : 0) * g.blocks + x_at;
    x[i] = *reinterpret_cast<const uint4*>(q + block * kBlock + (x_chunk & 1) * 16);
    e[i] = (uint8_t)exponents[block];
  };
  auto store_y = [&](bf16* stage, int i) {
    const int k = y_row + y_step(i);
    if constexpr (TERMS == 1) {
      *reinterpret_cast<uint4*>(stage + k * PY + y_chunk * 8) = make_uint4(y[i].w[0], y[i].w[1], y[i].w[2], y[i].w[3]);
    } else {
      // Each term is the leading 8 bits of what the terms before leave, cut
      // off, so the rest is exact.  The rests are taken of the value held to
      // finite numbers: an infinity stays one, and a NaN's first term (its
      // quiet bit set) is one.
      float first[8], v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        first[j] = __builtin_canonicalizef(value_of(y[i], j));
        v[j] = __builtin_amdgcn_fmed3f(first[j], -MOST, MOST);
      }
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) w[j / 2] = t == 0 ? pack(first[j], first[j + 1]) : pack(v[j], v[j + 1]);
        *reinterpret_cast<uint4*>(stage + (t * KB + k) * PY + y_chunk * 8) = make_uint4(w[0], w[1], w[2], w[3]);
        if (t + 1 < TERMS)
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] -= __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u);
      }
    }
  };
  auto store_x = [&](bf16* stage, int i) {
    const int k = x_row + i * (THREADS / CX), exponent = (int8_t)e[i];
    stored[i] = __ballot(held[i]);
    const float step = !held[i] ? 0.0f : exponent == kNotFinite ? NAN : pow2(exponent);
    const uint32_t in[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[2 * j] = pack((float)(int8_t)in[j] * step, (float)(int8_t)(in[j] >> 8) * step);
      w[2 * j + 1] = pack((float)(int8_t)(in[j] >> 16) * step, (float)(int8_t)(in[j] >> 24) * step);
    }
    bf16* to = stage + TERMS * KB * PY + k * PX + x_chunk * 16;
    *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    *reinterpret_cast<uint4*>(to + 8) = make_uint4(w[4], w[5], w[6], w[7]);
  };

  // A slot without a row is left out of dy as well: an infinity or a NaN times
  // the row's zeros would be a NaN.  The lanes that stored the slot's row know
  // whether there is one: the bits from 32 (i & 1) + CX (lane / CY) on.  Each
  // lane clears what it stored itself.  131,072 slots of 64 experts, 2,048 x
  // 2,048: 1.157 ms with this branch, 1.180 with masks in store_y, 1.145 with
  // neither.
  auto clear_y = [&](bf16* stage) {
    uint64_t all = ~0ull;
#pragma unroll
    for (int i = 0; i < NX; ++i) all &= stored[i];
    if (all == ~0ull) return;   // the same for the wave
#pragma unroll
    for (int i = 0; i < NY; ++i)
      if (!(stored[i >> 1] >> (32 * (i & 1) + CX * (lane / CY)) & 1))
        for (int t = 0; t < TERMS; ++t)
          *reinterpret_cast<uint4*>(stage + (t * KB + y_row + y_step(i)) * PY + y_chunk * 8) = make_uint4(0, 0, 0, 0);
  };

  // A lane's place in a transposing read: lanes 0-15 give four slots of 16
  // columns and get a column each; lanes 16-31 the next 16 columns, lanes
  // 32-63 the slots 8 further on.
  const int read_k = (lane >> 5) * 8 + ((lane & 15) >> 2), read_m = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
  const int wn = (wave / WC) * (BN / WN), wc = (wave % WC) * (BC / WC);
  auto fragment = [&](const bf16* from, int pitch) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 4 * pitch));
    const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
  };

  f32x16 acc[FC][FN] = {};
  // A step multiplies the tile at s0 from one half of the shared memory
  // while the next one goes from registers to the other half and the one
  // after that from memory to the registers, a slice of each between the
  // products of every 16 slots: conversions and addresses run in the shadow
  // of the matrix cores.  PLAIN: all of that lies inside the part.
  auto step = [&](int s0, const bf16* stage, bf16* next, auto plain_step) {
    constexpr bool PLAIN = decltype(plain_step)::value;
    constexpr int SLICES = KB / 16;
    const bool store = PLAIN || s0 + KB < it.to, load = PLAIN || s0 + 2 * KB < it.to;
    const bool plain = PLAIN || (y_wide && s0 + 3 * KB <= plain_to);
    const bf16* ys = stage + read_k * PY + wn + read_m;
    const bf16* xs = stage + TERMS * KB * PY + read_k * PX + wc + read_m;
#pragma unroll
    for (int h = 0; h < SLICES; ++h) {
      const int k = h * 16;
      bf16x8 a[FC];
#pragma unroll
      for (int i = 0; i < FC; ++i) a[i] = fragment(xs + k * PX + i * 32, PX);
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const bf16x8 b = fragment(ys + (t * KB + k) * PY + j * 32, PY);
#pragma unroll
          for (int i = 0; i < FC; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b, acc[i][j], 0, 0, 0);
        }
#pragma unroll
      for (int i = h * NY / SLICES; i < (h + 1) * NY / SLICES; ++i) {
        if (store) store_y(next, i);
        if (load) load_y(s0 + 2 * KB, i, plain);
      }
#pragma unroll
      for (int i = h * NX / SLICES; i < (h + 1) * NX / SLICES; ++i) {
        if (store) store_x(next, i);
        if (load) load_x(s0 + 2 * KB, i);
      }
    }
    if (load) load_rows(s0 + 3 * KB);
    if (store) clear_y(next);
    __syncthreads();
  };

  if (it.from < it.to) {
    auto load_all = [&](int s0) {
      for (int i = 0; i < NY; ++i) load_y(s0, i, y_wide && s0 + KB <= plain_to);
      for (int i = 0; i < NX; ++i) load_x(s0, i);
      load_rows(s0 + KB);
    };
    load_rows(it.from);
    load_all(it.from);
    for (int i = 0; i < NY; ++i) store_y(shared, i);
    for (int i = 0; i < NX; ++i) store_x(shared, i);
    clear_y(shared);
    if (it.from + KB < it.to) load_all(it.from + KB);
  }
  __syncthreads();
  int s0 = it.from;
  bf16 *stage = shared, *next = shared + STAGE;
  auto turn = [&] {
    bf16* was = stage;
    stage = next;
    next = was;
    s0 += KB;
  };
  if (y_wide)
    for (; s0 + 3 * KB <= plain_to; turn()) step(s0, stage, next, std::true_type{});
  for (; s0 < it.to; turn()) step(s0, stage, next, std::false_type{});

  // The tile leaves through shared memory, so that rows are written as whole
  // lines.  64 experts of 8 slots each, 2,048 x 2,048 in bfloat16 (537 MB):
  // 118 us, and 193 us when every lane wrote the four columns that it holds.
  auto write = [&](auto* out) {
    using D = std::remove_reference_t<decltype(*out)>;
    constexpr int V = 16 / sizeof(D), PITCH = BC + V;
    constexpr int FIT = 2 * STAGE * (int)sizeof(bf16) / (PITCH * (int)sizeof(D));
    constexpr int ROWS = FIT >= BN ? BN : FIT >= BN / 2 ? BN / 2 : BN / 4;   // of a pass
    static_assert(ROWS % 32 == 0 && ROWS <= FIT, "");
    D* tile = reinterpret_cast<D*>(shared);
    const bool wide = g.cols % V == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
#pragma unroll
    for (int first = 0; first < BN; first += ROWS) {
      if (first > 0) __syncthreads();
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = wn + j * 32 - first;
        if (n < 0 || n >= ROWS) continue;   // the same for a wave
#pragma unroll
        for (int i = 0; i < FC; ++i)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            struct alignas(4 * sizeof(D)) Four {
              D v[4];
            } four;
#pragma unroll
            for (int h = 0; h < 4; ++h) four.v[h] = (D)acc[i][j][r + h];
            *reinterpret_cast<Four*>(tile + (n + (lane & 31)) * PITCH + wc + i * 32 + r * 2 + (lane >> 5) * 4) = four;
          }
      }
      __syncthreads();
      if (wide) {
#pragma unroll 4
        for (int i = tid; i < ROWS * BC / V; i += THREADS) {
          const int row = i / (BC / V), c = i % (BC / V) * V, n = n0 + first + row;
          if (n < g.n && c0 + c < g.cols)
            *reinterpret_cast<uint4*>(out + (int64_t)n * g.cols + c0 + c) = *reinterpret_cast<const uint4*>(tile + row * PITCH + c);
        }
      } else {
#pragma unroll 4
        for (int i = tid; i < ROWS * BC; i += THREADS) {
          const int row = i / BC, c = i % BC, n = n0 + first + row;
          if (n < g.n && c0 + c < g.cols) out[(int64_t)n * g.cols + c0 + c] = tile[row * PITCH + c];
        }
      }
    }
  };
  if (it.partial < 0)
    write(dw + (int64_t)it.expert * g.n * g.cols);
  else
    write(partials + (int64_t)it.partial * g.n * g.cols);
}

constexpr int64_t kBlocksOfLaunch = 1 << 30;   // two threads each; a row has at most 2^15

// How a call's sums are cut, from its sizes alone.
Cut make_cut(int64_t experts, int64_t slots, int64_t n, int64_t cols, int32_t type) {
  Cut c{};
  // Tiles of 256 read half as much per product, those of 128 leave less over
  // at the edges of dW and of the parts: with 4,096 slots (times the terms of
  // dy) for each compute unit the larger ones are 14% faster, with 2,048 the
  // smaller ones 5%, with 512 26%.
  const int64_t terms = type == NETSIM_BF16 ? 1 : type == NETSIM_F16 ? 2 : 3;
  c.tile = slots * terms * ceil_div(n, 256) * ceil_div(cols, 256) / 256 >= 3000 ? 256 : 128;
  const int64_t tiles = ceil_div(n, c.tile) * ceil_div(cols, c.tile);   // of one expert
  // Steps of 64 slots keep a compute unit's shared memory to one workgroup,
  // those of 32 leave room for two or three smaller ones, which takes many
  // tiles to be of use.  16,384 slots in tiles of 128: with 512 tiles (8 experts
  // of 64) 69 us by 64 slots and 74 by 32, with 1,024 68 and 67, with 1,536 74 and
  // 68, with 4,096 119 and 115; 128 to 512 of 16 an expert 35 either way.  2,048
  // slots: up to 512 tiles 4% slower by 64, from 1,024 on 4 to 12%.
  c.step = terms == 1 && (c.tile == 256 || tiles * experts < 1024) ? 64 : 32;
  // the slots that each of the 256 compute units would have of one tile if
  // all were busy to the end; parts of a few steps cost more in partial sums
  // than they save
  c.longest = ceil_div(slots * tiles, 256);
  if (c.longest < 256) c.longest = 256;
  if (c.longest > kMaxSlots) c.longest = kMaxSlots;   // no sum is longer
  // joining the parts takes a launch more, about as long as 1,024 slots of one
  // tile, and a list of them another, which every wave's own search outweighs
  // with many experts or tiles.  16,384 slots, without a list and with one: 1, 4
  // and 8 experts of one tile 15.5 us and 18, 16 of them 16.6 and 18.2, 32 of
  // them 21.5 and 18.8; 1 expert of 16 tiles 28.7 and 30.6, 4 of them 34.9 and
  // 35.1, 8 of them 33.8 and 32.9, 8 of 64 tiles 70.6 and 69.4.
  c.plan = slots <= 1024 ? Cut::WHOLE : experts * tiles <= 64 && experts <= 16 ? Cut::BY_WAVE : Cut::LISTED;
  if (c.plan == Cut::WHOLE) return c;
  c.items = experts + slots / c.longest;
  c.joins = slots / c.longest < experts ? slots / c.longest : experts;
  c.partials = 2 * (slots / c.longest);
  c.bytes = 16 * (c.items + c.joins) + 4 * c.partials * n * cols;
  return c;
}

}  // namespace
}  // namespace netsim_ops

using namespace netsim_ops;

extern "C" netsim_status netsim_act_save(int32_t device, int64_t rows, int32_t cols, int32_t type, const void* d_x,
                                         int64_t ld_x, int8_t* d_q, int8_t* d_exponents, void* hip_stream) {
  const char* what = "act_save";
  return entry(what, device, [&] {
    if (!type_ok(type)) return fail(NETSIM_E_INVALID, what, "bad type");
    if (rows < 0 || cols < 1 || cols > kMaxCols) return fail(NETSIM_E_INVALID, what, "bad rows or cols");
    if (ld_x < cols) return fail(NETSIM_E_INVALID, what, "ld_x is below cols");
    if (rows == 0) return (netsim_status)NETSIM_OK;
    if (!d_x || !d_q || !d_exponents) return fail(NETSIM_E_INVALID, what, "NULL array");
    if (!aligned(d_x, type_size(type)) || !aligned(d_q, 16))
      return fail(NETSIM_E_INVALID, what, "d_x is not aligned to its type, or d_q to 16 bytes");
    const int blocks = (int)ceil_div(cols, kBlock);
    if (rows > ((int64_t)1 << 37) / blocks) return fail(NETSIM_E_INVALID, what, "more than 2^37 blocks of 32 columns");
    return launch(what, device, [&] {
      with_type(type, [&](auto t) {
        using T = decltype(t);
        in_launches(rows, kBlocksOfLaunch / blocks, [&](int64_t first, int64_t n) {
          hipLaunchKernelGGL(save_kernel<T>, dim3((unsigned)ceil_div(n * blocks, 128)), dim3(256), 0,
                             static_cast<hipStream_t>(hip_stream), n, cols, blocks,
                             static_cast<const T*>(d_x) + first * ld_x, ld_x, d_q + first * blocks * kBlock,
                             d_exponents + first * blocks);
        });
      });
    });
  });
}

extern "C" netsim_status netsim_act_restore(int32_t device, int64_t rows, int32_t cols, const int8_t* d_q,
                                            const int8_t* d_exponents, int32_t type, void* d_x, int64_t ld_x,
                                            void* hip_stream) {
  const char* what = "act_restore";
  return entry(what, device, [&] {
    if (!type_ok(type)) return fail(NETSIM_E_INVALID, what, "bad type");
    if (rows < 0 || cols < 1 || cols > kMaxCols) return fail(NETSIM_E_INVALID, what, "bad rows or cols");
    if (ld_x < cols) return fail(NETSIM_E_INVALID, what, "ld_x is below cols");
    if (rows == 0) return (netsim_status)NETSIM_OK;
    if (!d_x || !d_q || !d_exponents) return fail(NETSIM_E_INVALID, what, "NULL array");
    if (!aligned(d_x, type_size(type)) || !aligned(d_q, 16))
      return fail(NETSIM_E_INVALID, what, "d_x is not aligned to its type, or d_q to 16 bytes");
    const int blocks = (int)ceil_div(cols, kBlock);
    if (rows > ((int64_t)1 << 37) / blocks) return fail(NETSIM_E_INVALID, what, "more than 2^37 blocks of 32 columns");
    return launch(what, device, [&] {
      with_type(type, [&](auto t) {
        using T = decltype(t);
        in_launches(rows, kBlocksOfLaunch / blocks, [&](int64_t first, int64_t n) {
          hipLaunchKernelGGL(restore_kernel<T>, dim3((unsigned)ceil_div(n * blocks, 128)), dim3(256), 0,
                             static_cast<hipStream_t>(hip_stream), n, cols, blocks, d_q + first * blocks * kBlock,
                             d_exponents + first * blocks, static_cast<T*>(d_x) + first * ld_x, ld_x);
        });
      });
    });
  });
}

extern "C" int64_t netsim_act_weight_grad_work_bytes(int32_t experts, int64_t slots, int32_t n, int32_t cols,
                                                     int32_t type) {
  if (experts < 1 || experts > 1024 || slots < 0 || slots > kMaxSlots || n < 1 || n > kMaxCols || cols < 1 ||
      cols > kMaxCols || !type_ok(type))
    return -1;
  return make_cut(experts, slots, n, cols, type).bytes;
}

extern "C" netsim_status netsim_act_weight_grad(int32_t device, int32_t experts, int64_t slots, int32_t n,
                                                int32_t cols, int32_t type, const void* d_dy, int64_t ld_dy,
                                                int64_t rows, const int8_t* d_q, const int8_t* d_exponents,
                                                const int32_t* d_row_of_slot, const int32_t* d_offsets,
                                                int32_t out_type, void* d_dw, void* d_work, int64_t work_bytes,
                                                void* hip_stream) {
  const char* what = "act_weight_grad";
  return entry(what, device, [&] {
    if (!type_ok(type) || !type_ok(out_type)) return fail(NETSIM_E_INVALID, what, "bad type");
    const int64_t work = netsim_act_weight_grad_work_bytes(experts, slots, n, cols, type);
    if (work < 0)
      return fail(NETSIM_E_INVALID, what, "experts must be 1 .. 1024, n and cols 1 .. 2^20, slots 0 .. 2^31-4097");
    if (rows < 0) return fail(NETSIM_E_INVALID, what, "rows is below 0");
    if (ld_dy < n) return fail(NETSIM_E_INVALID, what, "ld_dy is below n");
    if (!d_offsets || !d_dw || (slots > 0 && !d_dy) || (rows > 0 && (!d_q || !d_exponents)))
      return fail(NETSIM_E_INVALID, what, "NULL array");
    if (work_bytes < work || (work > 0 && !d_work))
      return fail(NETSIM_E_INVALID, what, "the workspace is too small (netsim_act_weight_grad_work_bytes)");
    if (!aligned(d_dy, type_size(type)) || !aligned(d_dw, type_size(out_type)) || !aligned(d_q, 16) ||
        !aligned(d_row_of_slot, 4) || !aligned(d_offsets, 4) || !aligned(d_work, 16))
      return fail(NETSIM_E_INVALID, what, "an array is not aligned to its type, or d_q or d_work to 16 bytes");
    const Grad g{{experts, n, cols, (int)slots, cols % 4 == 0 && aligned(d_dw, 4 * type_size(out_type))},
                 (int)ceil_div(cols, kBlock), rows, ld_dy, d_row_of_slot ? -1 : 0};
    const Cut cut = make_cut(experts, slots, n, cols, type);
    return launch(what, device, [&] {
      with_type(type, [&](auto t) {
        with_type(out_type, [&](auto o) {
          using T = decltype(t);
          using O = decltype(o);
          constexpr int LONG = Terms<T>::value == 1 ? 64 : 32;
          hipStream_t s = static_cast<hipStream_t>(hip_stream);
          Item* items = static_cast<Item*>(d_work);
          Join* joins = reinterpret_cast<Join*>(items + cut.items);
          float* partials = reinterpret_cast<float*>(joins + cut.joins);
          if (cut.plan == Cut::LISTED)
            hipLaunchKernelGGL(plan_kernel, dim3(1), dim3((unsigned)ceil_div(experts, 64) * 64), 0, s, g, cut, d_offsets, items, joins);
          auto run = [&](auto kernel, int threads) {
            const int lds = 2 * 2 * cut.step * (Terms<T>::value + 1) * (cut.tile + 32);
            (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            hipLaunchKernelGGL(kernel,
                               dim3((unsigned)(ceil_div(n, cut.tile) * ceil_div(cols, cut.tile)),
                                    (unsigned)(cut.plan == Cut::WHOLE ? experts : cut.items)),
                               dim3(threads), lds, s, g, cut, items, static_cast<const T*>(d_dy), d_q, d_exponents,
                               d_row_of_slot ? d_row_of_slot : d_offsets, d_offsets, static_cast<O*>(d_dw), partials);
          };
          if (cut.tile == 256)
            run(grad_kernel<T, O, 256, 256, 2, 4, LONG>, 512);
          else
            run(cut.step == LONG ? grad_kernel<T, O, 128, 128, 2, 2, LONG> : grad_kernel<T, O, 128, 128, 2, 2, 32>, 256);
          if (cut.joins > 0) {
            // mostly there are few experts to join, or none: groups that find
            // nothing to do cost 4 us at 14,000 of them
            const int64_t groups = ceil_div((int64_t)n * cols, 256), most = cut.joins < 32 ? 4096 / cut.joins : 128;
            hipLaunchKernelGGL(join_kernel<O>, dim3((unsigned)(groups < most ? groups : most), (unsigned)cut.joins),
                               dim3(256), 0, s, g, cut, d_offsets, joins, partials, static_cast<O*>(d_dw));
          }
        });
      });
    });
  });
}
