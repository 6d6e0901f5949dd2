// What the device code of every translation unit of libbpd shares: bf16 bit patterns, buffer descriptors, reductions across the
// lanes of an MFMA operand's rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef unsigned short bf16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ __forceinline__ float bf2f(bf16_t v) { return __uint_as_float(((unsigned)v) << 16); }
__device__ __forceinline__ bf16_t f2bf(float f) { return __builtin_bit_cast(bf16_t, (__bf16)f); }      // round to nearest even (one instruction)
// An argument that only a kernel's end reads, loaded where this stands: left to itself the compiler loads it there, and the trip
// (0.2 .. 0.4 us) is exposed.
template <typename T> __device__ __forceinline__ T* arg_now(T* v) { asm volatile("" ::"s"(v)); return v; }
__device__ __forceinline__ unsigned cvt_pk_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
// Descriptor of `bytes` bytes from p (both the same for the whole wave): loads past the end return zeros without a memory
// access, so that rows beyond a block's last one cost nothing and need no branch.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ rsrc_t rsrc_of(const void* p, unsigned bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00027000); }
__device__ __forceinline__ u32x4 buf_load16(rsrc_t r, unsigned off, unsigned soff) { return __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, (int)soff, 0); }
template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<bf16_t>(bf16_t v) { return bf2f(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f<bf16_t>(float v) { return f2bf(v); }

__device__ __forceinline__ float wave_max(float v) {
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
// Sum and maximum over the four lanes l, l ^ 16, l ^ 32, l ^ 48 (one row of an MFMA operand), in all of them.  The swaps
// exchange every second 16-lane row (the upper half) of one register with the others (the lower half) of another: no trip
// through LDS.
__device__ __forceinline__ float sum_rows(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float max_rows(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// ... and over the whole wave: lanes of a 16-lane row first (data-parallel-primitive moves), then the rows
template <int CTRL> __device__ __forceinline__ float dpp_move(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true)); }
// (four lanes side by side: added as sum_rows() adds its four)
__device__ __forceinline__ float quad_sum(float v) {
  v += dpp_move<0xB1>(v);                        // quad_perm 1 0 3 2
  return v + dpp_move<0x4E>(v);                  // quad_perm 2 3 0 1
}
__device__ __forceinline__ float wave_sum(float v) {
  v = quad_sum(v);
  v += dpp_move<0x141>(v);                       // row_half_mirror
  v += dpp_move<0x140>(v);                       // row_mirror
  return sum_rows(v);
}

// Element (m, c) of activations [rows][K] as row_gemm_kernel reads them: the operands of its matrix instructions one behind the other, [row tile][k-step of 32][lane][8], whole row tiles.  (Taken
// as operands out of rows in memory, a load of 1 KB touches 64 lines, which the L1 looks up one by one: 64 cycles instead of 16: the queries, keys
// and values of 320 x 1024 10.6 us, packed 8.3, their first FFN layer 12.8, 9.8, an output projection 6.8, 5.9;  170 rows 8.9, 7.3;  8.5, 6.4;  5.3, 5.1.)
__device__ __forceinline__ size_t packed_at(long m, int c, int K) {
  return (size_t)(m & ~15l) * K + (c >> 5) * 512 + ((c >> 3) & 3) * 128 + (int)(m & 15) * 8 + (c & 7);
}

// A tree of up to 16 nodes in a word: four bits a node, its parent (of node 0, which follows the prefix, 15: the word is not 0, which stands for a chain)
__device__ __forceinline__ int tree_parent(unsigned long long tree, int i) { return (int)(tree >> (4 * i) & 15); }
__device__ __forceinline__ int tree_depth(unsigned long long tree, int i) {
  int e = 0;
  for (; i > 0; ++e) i = tree_parent(tree, i);   // (a parent comes before its children)
  return e;
}
