// The operators of an attention sublayer (rotate.hip, heads.hip, dropout.hip): launchers and what their kernels share.
// dtype: 0 = fp32, 1 = bf16.  All pointers are device memory; every sum is held in fp32.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/zgr.h"

namespace zgr {

struct bf16_bits { uint16_t bits; };
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {      // two conversions in one instruction, to nearest even
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16_bits x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ void put_float(float x, float* p) { *p = x; }
__device__ __forceinline__ void put_float(float x, bf16_bits* p) { p->bits = (uint16_t)pack_bf16(x, x); }

// N consecutive entries on any address: the hardware takes wide loads and stores that are not aligned.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Run { uint32_t w[N * sizeof(T) / 4]; };
template <typename T, int N> __device__ __forceinline__ void load_run(const T* p, float (&f)[N]) {
  const Run<T, N> r = *reinterpret_cast<const Run<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = sizeof(T) == 4 ? __uint_as_float(r.w[sizeof(T) == 4 ? i : 0]) : (i & 1 ? high_bf16(r.w[i / 2]) : low_bf16(r.w[i / 2]));
}
template <typename T, int N> __device__ __forceinline__ void store_run(T* p, const float (&f)[N]) {
  Run<T, N> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; ++i) r.w[i] = __float_as_uint(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) r.w[i / 2] = pack_bf16(f[i], f[i + 1]);
  }
  *reinterpret_cast<Run<T, N>*>(p) = r;
}

// out[c] = sum over p of part[p n + c], in the order of p within each of 32 interleaved runs and then of the runs: the same bits every time.
hipError_t launch_part_sums(const float* part, int parts, int n, float* out, hipStream_t s);

struct RotateArgs {
  zgr_rotation how;
  zgr_heads q, k, q_out, k_out;      // backward: q, k the inputs of the forward pass, q_out, k_out the gradients of its outputs
  zgr_heads dq, dk;                  // backward only: the gradients of q and k
  float* part;                       // backward only: rotate_parts(how) rows of 2 head_dim sums, or NULL
};
int        rotate_parts(const zgr_rotation& how);
hipError_t launch_norm_rotate(const RotateArgs& a, hipStream_t s);
hipError_t launch_norm_rotate_backward(const RotateArgs& a, hipStream_t s);

struct DropoutArgs {
  int32_t rows, cols, x_dtype, stream_dtype;
  int64_t x_row, residual_row, out_row;      // entries from a row to the next; backward: x is dx, out is dout
  void* x; const void* bias; const void* residual; void* out;
  uint32_t threshold, site, step, k0, k1;
  float scale;
  uint64_t first_row;
  float* part;                               // backward only: dropout_parts(rows, cols) rows of cols sums, or NULL
};
int        dropout_parts(int rows, int cols);
hipError_t launch_dropout_add(const DropoutArgs& a, hipStream_t s);
hipError_t launch_dropout_add_backward(const DropoutArgs& a, hipStream_t s);

struct AttentionArgs {
  zgr_attention how;
  zgr_heads q, k, v, out, dout, dq, dk, dv;
  float* lse;                        // [batch][n_head][n_q]
  void* dbias;
  unsigned char* workspace;
};
size_t     attention_workspace(const zgr_attention& how);
size_t     attention_backward_workspace(const zgr_attention& how);
hipError_t launch_heads_forward(const AttentionArgs& a, hipStream_t s);
hipError_t launch_heads_backward(const AttentionArgs& a, hipStream_t s);

// zgr_last_error(NULL) gets the message (api.hip)
zgr_status refuse(zgr_status st, const char* fmt, ...);

}  // namespace zgr
