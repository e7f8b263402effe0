// Penalties, biases and masks on logits, and their log-probabilities.
//
// A row is read once for its maximum and sum (kept together, the sum rescaled
// when the maximum grows) and once more where its log-probabilities are wanted.
// The few classes that a history or a bias list names are found through a table
// in LDS behind a filter of one bit per class number modulo 65536.
#include <hip/hip_runtime.h>

#include "lb_scorer.h"

namespace lb {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kFilterWords = 65536 / 32;

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__bf16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float as_float(_Float16 x) { return static_cast<float>(x); }

struct Slot {
  int32_t id;      // -1: empty
  int32_t count;   // occurrences in the history
  int32_t bias;    // place in the bias list + 1, 0: none
};

// The classes that the row's history and bias list name.  `slots` (a power of
// two, at least twice as many as there may be names; 0: no names at all)
struct Named {
  uint32_t* filter;
  Slot* table;
  int32_t slots;
  const float* bias;
};

__device__ __forceinline__ void put(const Named& N, int32_t id, int32_t count, int32_t bias) {
  atomicOr(&N.filter[(id & 65535) >> 5], 1u << (id & 31));
  uint32_t at = (static_cast<uint32_t>(id) * 2654435761u) & (N.slots - 1);
  for (;;) {
    const int32_t was = atomicCAS(&N.table[at].id, -1, id);
    if (was == -1 || was == id) break;
    at = (at + 1) & (N.slots - 1);
  }
  if (count) atomicAdd(&N.table[at].count, count);
  if (bias) atomicMax(&N.table[at].bias, bias);
}

__device__ __forceinline__ Named names(const LogitArgs& A, int64_t row, int32_t slots, uint32_t* shared) {
  Named N{shared, reinterpret_cast<Slot*>(shared + kFilterWords), slots, nullptr};
  if (!slots) return N;
  for (int i = threadIdx.x; i < kFilterWords; i += blockDim.x) N.filter[i] = 0;
  for (int i = threadIdx.x; i < slots; i += blockDim.x) N.table[i] = Slot{-1, 0, 0};
  __syncthreads();
  for (int i = threadIdx.x; i < A.r.history_width; i += blockDim.x) {
    const int32_t id = A.r.history[row * A.r.history_width + i];
    if (id >= 0 && id < A.classes) put(N, id, 1, 0);
  }
  const int64_t list = A.r.bias_per_row ? row * A.r.bias_width : 0;
  N.bias = A.r.bias_values + list;
  for (int i = threadIdx.x; i < A.r.bias_width; i += blockDim.x) {
    const int32_t id = A.r.bias_ids[list + i];
    if (id >= 0 && id < A.classes) put(N, id, 0, i + 1);
  }
  __syncthreads();
  return N;
}

__device__ __forceinline__ float adjusted(const LogitArgs& A, const Named& N, const uint32_t* mask, int32_t w, float x) {
  if (N.slots && (N.filter[(w & 65535) >> 5] >> (w & 31) & 1u)) {
    uint32_t at = (static_cast<uint32_t>(w) * 2654435761u) & (N.slots - 1);
    while (N.table[at].id != -1 && N.table[at].id != w) at = (at + 1) & (N.slots - 1);
    const Slot s = N.table[at];
    if (s.id == w) {
      if (s.count) {
        x = x > 0.0f ? x / A.r.repetition : x * A.r.repetition;
        x = x - A.r.presence - A.r.frequency * static_cast<float>(s.count);
      }
      if (s.bias) x += N.bias[s.bias - 1];
    }
  }
  if (A.r.temperature != 1.0f) x /= A.r.temperature;
  if (mask && !(mask[w >> 5] >> (w & 31) & 1u)) x = -__builtin_inff();
  return x;
}

__device__ __forceinline__ const uint32_t* mask_of(const LogitArgs& A, int64_t row) {
  if (!A.r.mask) return nullptr;
  const int64_t k = A.r.mask_row ? A.r.mask_row[row] : A.r.mask_rows == 1 ? 0 : row;
  return k >= 0 && k < A.r.mask_rows ? A.r.mask + k * ((A.classes + 31) / 32) : nullptr;
}

// (m, l): a maximum and the sum of exp2(log2(e) (z - m)); nothing yet: (-inf, 0)
struct Sum {
  float m, l;
};
// what exponents are taken relative to: an infinite maximum would make inf - inf of them
__device__ __forceinline__ float safe(float m) { return __builtin_isinf(m) ? 0.0f : m; }
__device__ __forceinline__ void add(Sum& a, float z) {
  const float m = fmaxf(a.m, z), base = safe(m);
  a.l = a.l * __builtin_amdgcn_exp2f((a.m - base) * kLog2e) + __builtin_amdgcn_exp2f((z - base) * kLog2e);
  a.m = m;
}
__device__ __forceinline__ void join(Sum& a, float m2, float l2) {
  const float m = fmaxf(a.m, m2), base = safe(m);
  a.l = a.l * __builtin_amdgcn_exp2f((a.m - base) * kLog2e) + l2 * __builtin_amdgcn_exp2f((m2 - base) * kLog2e);
  a.m = m;
}
__device__ __forceinline__ Sum block_sum(Sum s) {
  __shared__ float sm[4], sl[4];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float m2 = __shfl_xor(s.m, d), l2 = __shfl_xor(s.l, d);
    join(s, m2, l2);
  }
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s.m, sl[threadIdx.x >> 6] = s.l;
  __syncthreads();
  Sum t{sm[0], sl[0]};
#pragma unroll
  for (int w = 1; w < 4; ++w) join(t, sm[w], sl[w]);
  return t;
}
// The log-sum-exp as maximum and rest: z - lse is taken as (z - m) - rest, which
// stays right where m is so large that m + rest is m.
struct Lse {
  float m, rest;
};
__device__ __forceinline__ Lse log_sum(Sum s) { return {safe(s.m), s.l == 0.0f ? -__builtin_inff() : log2f(s.l) * kLn2}; }
__device__ __forceinline__ float log_prob(float z, Lse lse) { return z == -__builtin_inff() ? z : (z - lse.m) - lse.rest; }

__device__ __forceinline__ void finish(const LogitArgs& A, int64_t row, Lse lse, float zt) {
  if (A.lse) A.lse[row] = lse.m + lse.rest;
  if (!A.score) return;
  const int32_t t = A.target[row];
  A.score[row] = t < 0 ? 0.0f : t >= A.classes ? __builtin_nanf("") : log_prob(zt, lse);
}

// One part of a row: its sum, and the whole rest where the row has one part.
// The parts' sums are kept at part[row][split] = (m, l) and the target's z after
// them.
template <typename T>
__global__ __launch_bounds__(256) void k_logits(LogitArgs A, int32_t slots) {
  extern __shared__ uint32_t shared[];
  __shared__ float zt;
  const int64_t row = blockIdx.x / A.splits;
  const int32_t split = blockIdx.x % A.splits;
  const int32_t per = (A.classes + A.splits - 1) / A.splits;
  const int32_t lo = min(A.classes, split * per), hi = min(A.classes, lo + per);
  const T* src = static_cast<const T*>(A.logits) + row * A.stride;
  const uint32_t* mask = mask_of(A, row);
  const Named N = names(A, row, slots, shared);
  const int32_t target = A.score ? A.target[row] : -1;
  Sum s{-__builtin_inff(), 0.0f};
  for (int32_t w = lo + threadIdx.x; w < hi; w += 256) {
    const float z = adjusted(A, N, mask, w, as_float(src[w]));
    add(s, z);
    if (w == target) zt = z;
  }
  s = block_sum(s);  // its barrier also shows zt to all
  if (A.splits > 1) {
    float* at = A.part + 2 * blockIdx.x;
    if (threadIdx.x == 0) {
      at[0] = s.m, at[1] = s.l;
      if (target >= lo && target < hi) A.part[2 * A.rows * A.splits + row] = zt;
    }
    return;
  }
  const Lse lse = log_sum(s);
  if (threadIdx.x == 0) finish(A, row, lse, zt);
  if (!A.logprobs) return;
  float* dst = A.logprobs + row * A.out_stride;
  for (int32_t w = lo + threadIdx.x; w < hi; w += 256) {
    const float z = adjusted(A, N, mask, w, as_float(src[w]));
    dst[w] = log_prob(z, lse);
  }
}

// Rows of several parts: joins the sums, then writes the part's log-probabilities.
template <typename T>
__global__ __launch_bounds__(256) void k_logits_join(LogitArgs A, int32_t slots, int32_t groups) {
  extern __shared__ uint32_t shared[];
  const int64_t row = blockIdx.x / groups;
  const int32_t split = blockIdx.x % groups;
  Sum s{-__builtin_inff(), 0.0f};
  for (int32_t k = threadIdx.x; k < A.splits; k += 256) join(s, A.part[2 * (row * A.splits + k)], A.part[2 * (row * A.splits + k) + 1]);
  s = block_sum(s);
  const Lse lse = log_sum(s);
  if (split == 0 && threadIdx.x == 0) finish(A, row, lse, A.part[2 * A.rows * A.splits + row]);
  if (!A.logprobs) return;
  const int32_t per = (A.classes + groups - 1) / groups;
  const int32_t lo = min(A.classes, split * per), hi = min(A.classes, lo + per);
  const T* src = static_cast<const T*>(A.logits) + row * A.stride;
  const uint32_t* mask = mask_of(A, row);
  const Named N = names(A, row, slots, shared);
  float* dst = A.logprobs + row * A.out_stride;
  for (int32_t w = lo + threadIdx.x; w < hi; w += 256) {
    const float z = adjusted(A, N, mask, w, as_float(src[w]));
    dst[w] = log_prob(z, lse);
  }
}

template <typename T>
hipError_t run(const LogitArgs& A, hipStream_t st) {
  const int32_t ids = A.r.history_width + A.r.bias_width;
  int32_t slots = 0;
  if (ids)
    for (slots = 64; slots < 2 * ids; slots <<= 1) {
    }
  const size_t lds = slots ? kFilterWords * 4 + slots * sizeof(Slot) : 0;
  k_logits<T><<<dim3(static_cast<unsigned>(A.rows * A.splits)), 256, lds, st>>>(A, slots);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.splits == 1) return e;
  const int32_t groups = A.logprobs ? A.splits : 1;
  k_logits_join<T><<<dim3(static_cast<unsigned>(A.rows * groups)), 256, A.logprobs ? lds : 0, st>>>(A, A.logprobs ? slots : 0, groups);
  return hipGetLastError();
}

}  // namespace

int32_t logits_splits(int64_t rows, int32_t classes) {
  int64_t s = rows > 0 ? (512 + rows - 1) / rows : 1;
  s = s < classes / 1024 ? s : classes / 1024;
  return static_cast<int32_t>(s < 1 ? 1 : s);
}

hipError_t launch_logits(const LogitArgs& A, int dtype, hipStream_t st) {
  return dtype == LB_F32 ? run<float>(A, st) : dtype == LB_BF16 ? run<__bf16>(A, st) : run<_Float16>(A, st);
}

}  // namespace lb
