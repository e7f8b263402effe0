// Low-rank adapters beside a shared projection: out_i = y_i + s_a B_a (A_a x_i).
//
// Two launches: the rows' rank-sized products h = A x (summed in 32 bits over
// parts of d_in, each part's sum kept apart so that the order of addition is
// fixed), then out = y + s B h.  Both work on 16 rows at a time and, within them,
// on the distinct adapters one after the other with the other adapters' rows
// held at zero: rows of one request lie together, so a tile mostly has one
// adapter, and where each row has its own the weights of every row's adapter
// have to be read anyway.
#include <hip/hip_runtime.h>

#include "lb_scorer.h"

namespace lb {
namespace {

// Operands of one matrix step: KS inputs of 16 rows times 16 columns, `W` of them a lane.
template <typename T>
struct Step;
template <>
struct Step<__bf16> {
  static constexpr int KS = 32, W = 8;
  typedef bf16x8 V;
  static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Step<_Float16> {
  static constexpr int KS = 32, W = 8;
  typedef f16x8 V;
  static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Step<float> {
  static constexpr int KS = 16, W = 4;
  typedef f32x4 V;
  static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// The distinct adapters of a tile's rows, those of this workgroup's turn: calls
// f(adapter, whether this lane's row has it).
template <typename F>
__device__ __forceinline__ void each_adapter(int32_t id, int turn, int turns, F&& f) {
  uint32_t todo = static_cast<uint32_t>(__ballot(id >= 0)) & 0xFFFFu;
  for (int k = 0; todo; ++k) {
    const int32_t a = __builtin_amdgcn_readlane(id, __builtin_ctz(todo));
    todo &= ~static_cast<uint32_t>(__ballot(id == a));
    if (k % turns == turn) f(a, id == a);
  }
}

__device__ __forceinline__ int32_t adapter_of(const LoraArgs& A, int64_t row) {
  if (row >= A.rows) return -1;
  const int32_t a = A.adapter[row];
  return a >= 0 && a < A.n_adapters ? a : -1;
}

// h[part][row][rank] for 16 rows and one part of d_in; the wavefronts take every
// fourth step of it.
template <typename T, int RT>
__global__ __launch_bounds__(256) void k_lora_down(LoraArgs A) {
  using S = Step<T>;
  const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, j = lane >> 4;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + n;
  const int32_t k_lo = blockIdx.z * A.kspan, k_hi = min(A.d_in, k_lo + A.kspan);
  __shared__ float red[4][RT * 4][64];
  const T* x = static_cast<const T*>(A.x) + row * A.x_stride;
  each_adapter(adapter_of(A, row), blockIdx.y, gridDim.y, [&](int32_t a, bool mine) {
    const T* w = static_cast<const T*>(A.a) + static_cast<int64_t>(a) * A.rank * A.d_in;
    f32x4 acc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r] = f32x4{0, 0, 0, 0};
    for (int32_t k0 = k_lo + wave * S::KS; k0 < k_hi; k0 += 4 * S::KS) {
      const int32_t k = k0 + j * S::W;
      typename S::V xf{};
      if (mine && k < k_hi) xf = *reinterpret_cast<const typename S::V*>(x + k);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        typename S::V wf{};
        if (r * 16 + n < A.rank && k < k_hi)
          wf = *reinterpret_cast<const typename S::V*>(w + static_cast<int64_t>(r * 16 + n) * A.d_in + k);
        acc[r] = S::mul(wf, xf, acc[r]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][4 * r + i][lane] = acc[r][i];
    __syncthreads();
    if (mine) {
      float* h = A.h + (static_cast<int64_t>(blockIdx.z) * A.rows + row) * A.rank;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int at = 4 * r + wave, k = r * 16 + 4 * j + wave;
        if (k < A.rank) h[k] = red[0][at][lane] + red[1][at][lane] + red[2][at][lane] + red[3][at][lane];
      }
    }
  });
}

constexpr int kUpChannels = 256;  // channels of d_out a workgroup takes: 64 a wavefront, 32 at a time

// h as matrix operands.  In 16 bits it goes as its rounding and what that leaves
// (2^-17 of it for bf16, 2^-22 for fp16), side by side along the summed axis;
// fp16 is taken relative to the row's largest power of two, so that no h is out
// of its range.
template <typename T, int RT>
struct Down {
  typename Step<T>::V v[RT];
  float unit;
  __device__ __forceinline__ void load(const LoraArgs& A, int64_t row, bool mine, int j) {
    const int64_t part = A.rows * static_cast<int64_t>(A.rank);
    const float* h = A.h + row * A.rank;
    unit = 1.0f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int c = 0; c < RT; ++c) {
        const int k = c * 16 + j * 4;
        f32x4 x{0, 0, 0, 0};
        if (mine && k < A.rank)
          for (int z = 0; z < A.ksplit; ++z) x += *reinterpret_cast<const f32x4*>(h + z * part + k);
        v[c] = x;
      }
    } else {
      float x[RT][8], most = 0.0f;
#pragma unroll
      for (int c = 0; c < RT; ++c) {
        const int q = c * 32 + j * 8, k = q < A.rank ? q : q - A.rank;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = 0.0f;
        if (mine && k < A.rank)
          for (int z = 0; z < A.ksplit; ++z) {
            float y[8];
            load8(h + z * part + k, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[c][i] += y[i];
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[c][i]));
      }
      if constexpr (__is_same(T, _Float16)) {
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const int32_t e = min(max(static_cast<int32_t>(__float_as_uint(most) >> 23), 2), 252);
        unit = __uint_as_float(static_cast<uint32_t>(e) << 23);
        const float inv = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
#pragma unroll
        for (int c = 0; c < RT; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[c][i] *= inv;
      }
#pragma unroll
      for (int c = 0; c < RT; ++c) {
        const bool low = c * 32 + j * 8 >= A.rank;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const T hi = static_cast<T>(x[c][i]);
          v[c][i] = low ? (__builtin_isinf(x[c][i]) ? T(0.0f) : static_cast<T>(x[c][i] - static_cast<float>(hi))) : hi;
        }
      }
    }
  }
};

template <typename T, int RT>
__global__ __launch_bounds__(256) void k_lora_up(LoraArgs A) {
  using S = Step<T>;
  const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, j = lane >> 4;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + n;
  const int32_t o_lo = blockIdx.z * kUpChannels + wave * (kUpChannels / 4);
  const int32_t id = adapter_of(A, row);
  if (blockIdx.y == 0 && id < 0 && row < A.rows && (A.out != A.y)) {
    for (int32_t o = o_lo + j * 8; o < min(o_lo + kUpChannels / 4, A.d_out); o += 32) {
      float x[8];
      load8(static_cast<const T*>(A.y) + row * A.y_stride + o, x);
      store8(static_cast<T*>(A.out) + row * A.out_stride + o, x);
    }
  }
  each_adapter(id, blockIdx.y, gridDim.y, [&](int32_t a, bool mine) {
    Down<T, RT> h;
    h.load(A, row, mine, j);
    const float scale = (A.scale ? A.scale[a] : 1.0f) * h.unit;
    const T* w = static_cast<const T*>(A.b) + static_cast<int64_t>(a) * A.d_out * A.rank;
#pragma unroll
    for (int g = 0; g < kUpChannels / 128; ++g) {
      const int32_t o0 = o_lo + g * 32;
      if (o0 >= A.d_out) break;
      f32x4 acc[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // row m of the operand is channel 8 (m / 4) + 4 u + m % 4, so that a lane gets eight adjacent ones
        const int32_t o = o0 + (n >> 2) * 8 + u * 4 + (n & 3);
        acc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < RT; ++c) {
          const int q = c * S::KS + j * S::W, k = q < A.rank ? q : q - A.rank;
          typename S::V wf{};
          if (o < A.d_out && k < A.rank && (sizeof(T) == 2 || q < A.rank))
            wf = *reinterpret_cast<const typename S::V*>(w + static_cast<int64_t>(o) * A.rank + k);
          acc[u] = S::mul(wf, h.v[c], acc[u]);
        }
      }
      const int32_t o = o0 + j * 8;
      if (mine && o < A.d_out) {
        float x[8];
        load8(static_cast<const T*>(A.y) + row * A.y_stride + o, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = fmaf(scale, acc[0][i], x[i]);
          x[4 + i] = fmaf(scale, acc[1][i], x[4 + i]);
        }
        store8(static_cast<T*>(A.out) + row * A.out_stride + o, x);
      }
    }
  });
}

template <typename T, int RT>
hipError_t run(const LoraArgs& A, hipStream_t st) {
  const unsigned tiles = static_cast<unsigned>((A.rows + 15) / 16);
  const unsigned chunks = static_cast<unsigned>((A.d_out + kUpChannels - 1) / kUpChannels);
  // few tiles: the adapters of a tile side by side
  const unsigned down = tiles * A.ksplit < 512 ? 16 : 1, up = static_cast<int64_t>(tiles) * chunks < 512 ? 16 : 1;
  k_lora_down<T, RT><<<dim3(tiles, down, static_cast<unsigned>(A.ksplit)), 256, 0, st>>>(A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_lora_up<T, RT><<<dim3(tiles, up, chunks), 256, 0, st>>>(A);
  return hipGetLastError();
}

template <typename T>
hipError_t by_rank(const LoraArgs& A, hipStream_t st) {
  return A.rank <= 16 ? run<T, 1>(A, st) : A.rank <= 32 ? run<T, 2>(A, st) : A.rank <= 64 ? run<T, 4>(A, st) : run<T, 8>(A, st);
}

}  // namespace

int32_t lora_ksplit(int64_t rows, int32_t d_in, int32_t* kspan) {
  const int64_t tiles = (rows + 15) / 16;
  int64_t s = tiles > 0 ? (512 + tiles - 1) / tiles : 1;
  s = s < d_in / 256 ? s : d_in / 256;
  s = s < 1 ? 1 : s > 8 ? 8 : s;
  *kspan = static_cast<int32_t>(((d_in + s - 1) / s + 127) / 128 * 128);
  return (d_in + *kspan - 1) / *kspan;
}

hipError_t launch_lora(const LoraArgs& A, int dtype, hipStream_t st) {
  return dtype == LB_F32 ? by_rank<float>(A, st) : dtype == LB_BF16 ? by_rank<__bf16>(A, st) : by_rank<_Float16>(A, st);
}

}  // namespace lb
