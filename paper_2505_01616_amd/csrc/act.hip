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

namespace netsim_ops {
namespace {

constexpr int kBlock = 32;          // columns that share an exponent
constexpr int kNotFinite = -128;    // exponent of a block that held an infinity or a NaN

// 2^e as a float, -126 <= e <= 127.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// ----------------------------------------------------------- save, restore
// Four lanes per block, eight columns each.
template <class T>
__global__ __launch_bounds__(256) void save_kernel(int64_t rows, int cols, int blocks, const T* __restrict__ x,
                                                   int64_t ld, int8_t* __restrict__ q, int8_t* __restrict__ exponents) {
  const int64_t n = rows * blocks * 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t block = i >> 2, row = block / blocks;
    const int at = (int)(block % blocks), col = at * kBlock + ((int)i & 3) * 8;
    const T* from = x + row * ld + col;
    float v[8], top = 0.0f;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = col + j < cols ? (float)from[j] : 0.0f;
      odd |= !isfinite(v[j]);
      top = fmaxf(top, fabsf(v[j]));
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      top = fmaxf(top, __shfl_xor(top, o, 64));
      odd |= __shfl_xor((int)odd, o, 64) != 0;
    }
    int e = (int)(__float_as_uint(top) >> 23) - 127 - 6;
    e = e < -126 ? -126 : e;
    // 2^-e as two factors: -e reaches 126, and a subnormal needs no more
    const float up = pow2(-e);
    uint32_t word[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float r = odd ? 0.0f : fminf(fmaxf(rintf(v[j] * up), -127.0f), 127.0f);
      word[j >> 2] |= (uint32_t)(uint8_t)(int8_t)(int)r << (8 * (j & 3));
    }
    *reinterpret_cast<uint2*>(q + i * 8) = make_uint2(word[0], word[1]);
    if ((i & 3) == 0) exponents[block] = odd ? (int8_t)kNotFinite : (int8_t)e;
  }
}

template <class T>
__global__ __launch_bounds__(256) void restore_kernel(int64_t rows, int cols, int blocks,
                                                      const int8_t* __restrict__ q,
                                                      const int8_t* __restrict__ exponents, T* __restrict__ x,
                                                      int64_t ld) {
  const int64_t n = rows * blocks * 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t block = i >> 2, row = block / blocks;
    const int at = (int)(block % blocks), col = at * kBlock + ((int)i & 3) * 8;
    const int e = exponents[block];
    const float step = e == kNotFinite ? NAN : pow2(e);
    T* to = x + row * ld + col;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j < cols) to[j] = (T)((float)q[i * 8 + j] * step);
  }
}

// --------------------------------------------------------- weight gradient
// dW[e][n][c] = sum over the slots s of expert e of dy[s][n] x[row(s)][c].
// A workgroup per 128 x 128 tile of one expert's gradient; a step takes 32
// slots through shared memory.  dy enters the matrix cores as bfloat16: one
// term for bfloat16, two for float16 and three for float32, whose sum is the
// value without rounding (down to bfloat16's smallest magnitude).
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f32x16 = __attribute__((ext_vector_type(16))) float;

struct Grad {
  int experts, n, cols, blocks;
  int64_t slots, rows, ld;
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

// The leading 8 significant bits of y, the rest cut off (never an overflow,
// and the rest is exact); a NaN stays one.
__device__ __forceinline__ float top_bits(float y) {
  uint32_t b = __float_as_uint(y);
  b |= isnan(y) ? 0x400000u : 0u;
  return __uint_as_float(b & 0xffff0000u);
}

// The bounds of an expert's slots, held to the arrays.
__device__ __forceinline__ void segment(const int32_t* offsets, int e, int64_t slots, int64_t* from, int64_t* to) {
  const int64_t a = offsets[e], b = offsets[e + 1];
  *from = a < 0 ? 0 : a > slots ? slots : a;
  *to = b < *from ? *from : b > slots ? slots : b;
}

template <class T, class O>
__global__ __launch_bounds__(256) void grad_kernel(Grad g, const T* __restrict__ dy, const int8_t* __restrict__ q,
                                                   const int8_t* __restrict__ exponents,
                                                   const int32_t* __restrict__ row_of_slot,
                                                   const int32_t* __restrict__ offsets, O* __restrict__ dw) {
  constexpr int TERMS = Terms<T>::value, K = 32, PITCH = K + 8;
  __shared__ __align__(16) bf16 y_tile[TERMS][128 * PITCH];  // [n][slot]
  __shared__ __align__(16) bf16 x_tile[128 * PITCH];         // [column][slot]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int e = blockIdx.z, n0 = blockIdx.y * 128, c0 = blockIdx.x * 128;
  int64_t from, to;
  segment(offsets, e, g.slots, &from, &to);
  f32x16 acc[2][2] = {};
  for (int64_t s0 = from; s0 < to; s0 += K) {
    __syncthreads();
    for (int i = tid; i < K * 128; i += 256) {
      const int k = i >> 7, m = i & 127;
      const int64_t s = s0 + k;
      float y = s < to && n0 + m < g.n ? (float)dy[s * g.ld + n0 + m] : 0.0f;
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        const float part = top_bits(y);
        y_tile[t][m * PITCH + k] = (bf16)part;
        y = isfinite(y) ? y - part : 0.0f;
      }
      const int64_t row = s < to ? row_of_slot ? row_of_slot[s] : s : -1;
      float x = 0.0f;
      if (row >= 0 && row < g.rows && c0 + m < g.cols) {
        const int p = exponents[row * g.blocks + (c0 + m) / kBlock];
        x = (float)q[row * g.blocks * kBlock + c0 + m] * (p == kNotFinite ? NAN : pow2(p));
      }
      x_tile[m * PITCH + k] = (bf16)x;
    }
    __syncthreads();
    const int wn = (wave >> 1) * 64, wc = (wave & 1) * 64;
#pragma unroll
    for (int k = 0; k < K; k += 16) {
      const int kk = k + (lane >> 5) * 8;
      bf16x8 b[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) b[j] = *reinterpret_cast<bf16x8*>(&x_tile[(wc + j * 32 + (lane & 31)) * PITCH + kk]);
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bf16x8 a = *reinterpret_cast<bf16x8*>(&y_tile[t][(wn + i * 32 + (lane & 31)) * PITCH + kk]);
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b[j], acc[i][j], 0, 0, 0);
        }
    }
  }
  O* out = dw + (int64_t)e * g.n * g.cols;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = n0 + (wave >> 1) * 64 + i * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
        const int c = c0 + (wave & 1) * 64 + j * 32 + (lane & 31);
        if (n < g.n && c < g.cols) out[(int64_t)n * g.cols + c] = (O)acc[i][j][r];
      }
}

constexpr int kMaxCols = 1 << 20;

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
    return launch(what, device, [&] {
      const int64_t groups = ceil_div(rows * blocks * 4, 256);
      with_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(save_kernel<T>, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0,
                           static_cast<hipStream_t>(hip_stream), rows, cols, blocks, static_cast<const T*>(d_x), ld_x,
                           d_q, d_exponents);
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
    return launch(what, device, [&] {
      const int64_t groups = ceil_div(rows * blocks * 4, 256);
      with_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(restore_kernel<T>, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0,
                           static_cast<hipStream_t>(hip_stream), rows, cols, blocks, d_q, d_exponents,
                           static_cast<T*>(d_x), ld_x);
      });
    });
  });
}

extern "C" int64_t netsim_act_weight_grad_work_bytes(int32_t experts, int64_t slots, int32_t n, int32_t cols,
                                                     int32_t type) {
  if (experts < 1 || experts > 1024 || slots < 0 || slots > 0x7fffffff || n < 1 || n > kMaxCols || cols < 1 ||
      cols > kMaxCols || !type_ok(type))
    return -1;
  return 0;
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
      return fail(NETSIM_E_INVALID, what, "experts must be 1 .. 1024, n and cols 1 .. 2^20, slots 0 .. 2^31-1");
    if (rows < 0) return fail(NETSIM_E_INVALID, what, "rows is below 0");
    if (ld_dy < n) return fail(NETSIM_E_INVALID, what, "ld_dy is below n");
    if (!d_offsets || !d_dw || (slots > 0 && !d_dy) || (rows > 0 && (!d_q || !d_exponents)))
      return fail(NETSIM_E_INVALID, what, "NULL array");
    if (work_bytes < work || (work > 0 && !d_work))
      return fail(NETSIM_E_INVALID, what, "the workspace is too small (netsim_act_weight_grad_work_bytes)");
    if (!aligned(d_dy, type_size(type)) || !aligned(d_dw, type_size(out_type)) || !aligned(d_q, 16) ||
        !aligned(d_row_of_slot, 4) || !aligned(d_offsets, 4) || !aligned(d_work, 16))
      return fail(NETSIM_E_INVALID, what, "an array is not aligned to its type, or d_q or d_work to 16 bytes");
    const Grad g{experts, n, cols, (int)ceil_div(cols, kBlock), slots, rows, ld_dy};
    return launch(what, device, [&] {
      with_type(type, [&](auto t) {
        with_type(out_type, [&](auto o) {
          using T = decltype(t);
          using O = decltype(o);
          hipLaunchKernelGGL((grad_kernel<T, O>), dim3((unsigned)ceil_div(cols, 128), (unsigned)ceil_div(n, 128), experts),
                             dim3(256), 0, static_cast<hipStream_t>(hip_stream), g, static_cast<const T*>(d_dy), d_q,
                             d_exponents, d_row_of_slot, d_offsets, static_cast<O*>(d_dw));
        });
      });
    });
  });
}
