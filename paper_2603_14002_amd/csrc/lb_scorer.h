// The fusion scorer's operators: launchers (host) and what their kernels share
// (device).  Defined in lb_kv.hip, lb_logits.hip and lb_lora.hip, called by
// lb_scorer_api.cpp after every argument has been checked.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/lightbeam_scorer.h"

namespace lb {

// a ragged batch and its cache, as the kernels take them
struct KvArgs {
  uint8_t* pages;
  int64_t n_pages;
  uint32_t* flags;
  const int32_t* starts;
  const int32_t* lengths;
  const int32_t* table;
  int32_t n_seqs, n_rows, max_pages, max_new;
  int32_t page_shift;  // log2 of the page's tokens
  int32_t kv_heads, q_heads;
};

struct AppendArgs {
  KvArgs kv;
  const void *q, *k, *v;
  void* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const float *cos, *sin;
  int32_t positions, rot, interleaved;
};

struct ReadArgs {
  KvArgs kv;
  void *k, *v;
  int64_t k_stride, v_stride;
};

struct AttendArgs {
  KvArgs kv;
  const void* q;
  void* out;
  int64_t q_stride, out_stride;
  float* lse;
  float* part;  // partial sums of split key ranges (see lb_kv.hip)
  float scale2;  // scale * log2(e)
  int32_t window;
  // the plan's
  int32_t tiles, splits, part_rows;
  uint32_t few_units, jobs;
  int64_t units, part_sums;
  int32_t few_rows;
  bool alone;
};

struct LoraArgs {
  const void *x, *y, *a, *b;
  void* out;
  const int32_t* adapter;
  const float* scale;
  float* h;
  int64_t x_stride, y_stride, out_stride;
  int32_t rows, d_in, d_out, rank, n_adapters;
  bool whole;  // in one launch
};

struct LogitArgs {
  const void* logits;
  int64_t stride;
  float* logprobs;
  int64_t out_stride;
  const int32_t* target;
  float *score, *lse, *part;
  int64_t rows, row0;  // row0: the launch's first row
  int32_t classes, splits;
  lb_logit_rules r;
};

// How an attention call is cut up (see attend_plan).  Few-row kernel: the query rows
// of a sequence and KV head up to which it takes them (0: it does not run), tiles of
// 16 rows, their units if they are numbered by the rows there are (else 0), jobs in
// all, whether a wavefront takes one alone, the parts that a key range is cut
// into, the rows of a tile whose parts are kept, the floats of these and where the
// parts' sums start among them.  Many-row kernel: its units of rows, 0: none.  groups:
// the most workgroups that a launch would have, of any type.
struct AttendPlan {
  int32_t few_rows;
  bool alone;
  int32_t tiles, splits, part_rows;
  int64_t few_units, jobs;
  int64_t part_floats, part_sums, units, groups;
};
AttendPlan attend_plan(const KvArgs& kv, int head_dim, int dtype);  // part_floats and groups are the same for every type

hipError_t launch_kv_append(const AppendArgs& A, int head_dim, int dtype, hipStream_t st);
hipError_t launch_kv_read(const ReadArgs& A, int head_dim, int dtype, hipStream_t st);
hipError_t launch_kv_attend(const AttendArgs& A, int head_dim, int dtype, hipStream_t st);

// the call is one launch, and needs no workspace (if out and x have no memory in common)
bool lora_whole(int64_t rows, int32_t d_in, int32_t d_out, int32_t rank);
hipError_t launch_lora(const LoraArgs& A, int dtype, hipStream_t st);

// parts of a row that its sum is taken over (1: no workspace)
int32_t logits_splits(int64_t rows, int32_t classes);
hipError_t launch_logits(const LogitArgs& A, int dtype, hipStream_t st);

#ifdef __HIPCC__

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// the wavefront's index in its workgroup, in a scalar register: what follows from it is uniform
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// eight consecutive values from 16-B aligned memory, as 32-bit floats
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const _Float16* p, float (&x)[8]) {
  const f16x8 w = *reinterpret_cast<const f16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(w[i]);
}

// eight consecutive values to 16-B aligned memory, each rounded to nearest
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = static_cast<__bf16>(x[i]);
  *reinterpret_cast<bf16x8*>(p) = w;
}
__device__ __forceinline__ void store8(_Float16* p, const float (&x)[8]) {
  f16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = static_cast<_Float16>(x[i]);
  *reinterpret_cast<f16x8*>(p) = w;
}

// The same for what is read once and what is not read again soon: it does not
// push other data out of the caches.
__device__ __forceinline__ void load8_nt(const float* p, float (&x)[8]) {
  const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
__device__ __forceinline__ void load8_nt(const __bf16* p, float (&x)[8]) {
  const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8_nt(const _Float16* p, float (&x)[8]) {
  const f16x8 w = __builtin_nontemporal_load(reinterpret_cast<const f16x8*>(p));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(w[i]);
}

__device__ __forceinline__ void store8_nt(float* p, const float (&x)[8]) {
  __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, reinterpret_cast<f32x4*>(p + 4));
}
__device__ __forceinline__ void store8_nt(__bf16* p, const float (&x)[8]) {
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = static_cast<__bf16>(x[i]);
  __builtin_nontemporal_store(w, reinterpret_cast<bf16x8*>(p));
}
__device__ __forceinline__ void store8_nt(_Float16* p, const float (&x)[8]) {
  f16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = static_cast<_Float16>(x[i]);
  __builtin_nontemporal_store(w, reinterpret_cast<f16x8*>(p));
}

// x rounded to bf16, but finite, so that the rest of it can be taken: that of an
// infinity (NaN) is an infinity (NaN) then
__device__ __forceinline__ __bf16 first_piece(float x) {
  const float largest = __uint_as_float(0x7F7F0000u);
  return static_cast<__bf16>(__builtin_amdgcn_fmed3f(x, -largest, largest));
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

#endif  // __HIPCC__

}  // namespace lb
