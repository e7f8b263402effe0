// Low-rank adapters beside a shared projection: out_i = y_i + s_a B_a (A_a x_i).
//
// Two launches: the rows' rank-sized products h = A x, kept in 32 bits, then out =
// y + s B h (one for few rows and small weights).  Both work on 16 rows at a time
// and, within them, on the distinct adapters with the other adapters' rows held at zero: rows of one request lie together, so a tile mostly has one
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

// A wavefront's share of h = A x for 16 rows and the rank's entries r0 .. r0 + 16 RT
// - 1 (rows not `mine`: zero): every W-th piece of d_in.  A piece is two matrix
// steps: a lane takes 32 adjacent bytes of its row, so that the four lanes of a row
// read whole lines of 128 B.  U pieces are on their way at a time.
template <typename T, int RT, int W>
__device__ __forceinline__ void down_share(const LoraArgs& A, const T* x, int32_t a, int32_t r0, bool mine, int wave, int n, int j, f32x4 (&acc)[RT]) {
  using S = Step<T>;
  constexpr int U = RT <= 2 ? 4 : 2, KS = 2 * S::KS;
  const T* w = static_cast<const T*>(A.a) + (static_cast<int64_t>(a) * A.rank + r0 + n) * A.d_in;
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[r] = f32x4{0, 0, 0, 0};
  for (int32_t k0 = wave * KS; k0 < A.d_in; k0 += U * W * KS) {
    typename S::V xf[U][2], wf[U][2][RT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const int32_t k = k0 + u * W * KS + (2 * j + v) * S::W;
        xf[u][v] = typename S::V{};
        if (mine && k < A.d_in) xf[u][v] = *reinterpret_cast<const typename S::V*>(x + k);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          wf[u][v][r] = typename S::V{};
          if (r0 + r * 16 + n < A.rank && k < A.d_in)
            wf[u][v][r] = *reinterpret_cast<const typename S::V*>(w + static_cast<int64_t>(r * 16) * A.d_in + k);
        }
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r] = S::mul(wf[u][v][r], xf[u][v], acc[r]);
  }
}

// Joins the wavefronts' shares in LDS: put(k, sum) for entry k of the lane's row.
template <int RT, int W, typename F>
__device__ __forceinline__ void down_join(float (&red)[W][RT * 4][64], const f32x4 (&acc)[RT], int wave, int lane, F&& put) {
  __syncthreads();  // the last adapter's sums have been read
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[wave][4 * r + i][lane] = acc[r][i];
  __syncthreads();
  for (int at = wave; at < RT * 4; at += W) {
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) sum += red[k][at][lane];
    put((at >> 2) * 16 + 4 * (lane >> 4) + (at & 3), sum);
  }
}

// 8192 x 4096 in bf16, rank 16: 23 us, 2.9 TB/s, as long as a plain sum over these rows
// takes (22 us).
constexpr int kDownWaves = 8;  // 64 KB of LDS at most

template <typename T, int RT>
__global__ __launch_bounds__(64 * kDownWaves) void k_lora_down(LoraArgs A) {
  constexpr int W = kDownWaves;
  const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, j = lane >> 4;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + n;
  const int32_t r0 = static_cast<int32_t>(blockIdx.z) * (16 * RT);  // the first of the workgroup's entries of the rank
  __shared__ float red[W][RT * 4][64];
  const T* x = static_cast<const T*>(A.x) + row * A.x_stride;
  each_adapter(adapter_of(A, row), blockIdx.y, gridDim.y, [&](int32_t a, bool mine) {
    f32x4 acc[RT];
    down_share<T, RT, W>(A, x, a, r0, mine, wave, n, j, acc);
    down_join<RT, W>(red, acc, wave, lane, [&](int k, float sum) {
      if (mine && r0 + k < A.rank) A.h[row * A.rank + r0 + k] = sum;
    });
  });
}

constexpr int kUpChannels = 256;  // channels of d_out a workgroup takes: 64 a wavefront

// h of a row as matrix operands.  In 16 bits it goes as its rounding and what that
// leaves (2^-16 of it for bf16, 2^-22 for fp16): two products with the same
// weights, or, up to rank 16, side by side along the summed axis of one product.
// fp16 is taken relative to the row's largest power of two, so that no h is out of
// its range.
template <typename T, int RT>
struct Down {
  using S = Step<T>;
  static constexpr bool wide = sizeof(T) == 4, paired = !wide && RT == 1;
  static constexpr int N = wide ? RT : paired ? 1 : RT / 2;  // products along the rank
  static constexpr int pieces = wide || paired ? 1 : 2;
  typename S::V v[pieces][N];
  float unit;

  // the first of the rank's entries that the lane has in product c (past the rank: none)
  static __device__ __forceinline__ int32_t entry(int c, int j, int32_t rank) {
    const int32_t q = c * S::KS + j * S::W;
    return paired && q >= rank ? (q < 2 * rank ? q - rank : rank) : q;
  }

  __device__ __forceinline__ void load(const LoraArgs& A, const float* h, bool mine, int j) {
    unit = 1.0f;
    if constexpr (wide) {
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const int32_t k = entry(c, j, A.rank);
        v[0][c] = f32x4{0, 0, 0, 0};
        if (mine && k < A.rank) v[0][c] = *reinterpret_cast<const f32x4*>(h + k);
      }
    } else {
      float x[N][8], most = 0.0f;
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const int32_t k = entry(c, j, A.rank);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = 0.0f;
        if (mine && k < A.rank) load8(h + k, x[c]);
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
        for (int c = 0; c < N; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[c][i] *= inv;
      }
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const bool second = paired && c * S::KS + j * S::W >= A.rank;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          T hi, lo;
          if constexpr (__is_same(T, __bf16)) {
            hi = first_piece(x[c][i]);
            lo = static_cast<T>(x[c][i] - static_cast<float>(hi));
          } else {
            // an infinity is one piece: the rest of it would be NaN
            hi = static_cast<T>(x[c][i]);
            lo = __builtin_isinf(x[c][i]) ? T(0.0f) : static_cast<T>(x[c][i] - static_cast<float>(hi));
          }
          v[0][c][i] = second ? lo : hi;
          if constexpr (pieces == 2) v[1][c][i] = lo;
        }
      }
    }
  }
};

// out = y + s B h.  whole: h is computed here too, by each workgroup for its own
// channels, else k_lora_down has left it in the workspace.  8192 x 6144 in bf16, rank
// 16: 44 us, 4.5 TB/s (a plain elementwise kernel: 36); 128 rows of their own adapters,
// rank 64, 8192 channels: 30 us, 4.0 TB/s of weights.  Bound by memory.
template <typename T, int RT, bool whole>
__global__ __launch_bounds__(256) void k_lora_up(LoraArgs A) {
  using S = Step<T>;
  using H = Down<T, RT>;
  constexpr int G = kUpChannels / 128;  // pairs of 16-channel tiles a wavefront
  const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, j = lane >> 4;
  const uint32_t chunks = (A.d_out + kUpChannels - 1) / kUpChannels;  // side by side: rows are streamed
  const int64_t row = static_cast<int64_t>(blockIdx.x / chunks) * 16 + n;
  const int32_t o_lo = blockIdx.x % chunks * kUpChannels + wave * (kUpChannels / 4);
  // A lane has the channels o_lo + 32 g + 8 j .. + 7 of its row (32 bits: 4 j .. + 3
  // of both 16): the four lanes of a row read and write 64 adjacent bytes at a time.
  const T* src = static_cast<const T*>(A.y) + row * A.y_stride;
  T* dst = static_cast<T*>(A.out) + row * A.out_stride;
  const auto load = [&](float (&y)[8], int g) {
    const int32_t o = o_lo + 32 * g;
    if constexpr (H::wide) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 v{0, 0, 0, 0};
        if (o + 16 * u + 4 * j < A.d_out) v = *reinterpret_cast<const f32x4*>(src + o + 16 * u + 4 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[4 * u + i] = v[i];
      }
    } else if (o + 8 * j < A.d_out) {
      load8(src + o + 8 * j, y);
    }
  };
  const auto store = [&](const float (&y)[8], int g) {
    const int32_t o = o_lo + 32 * g;
    if constexpr (H::wide) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (o + 16 * u + 4 * j < A.d_out)
          *reinterpret_cast<f32x4*>(dst + o + 16 * u + 4 * j) = f32x4{y[4 * u], y[4 * u + 1], y[4 * u + 2], y[4 * u + 3]};
    } else if (o + 8 * j < A.d_out) {
      store8(dst + o + 8 * j, y);
    }
  };
  float y[G][8];
  __shared__ float red[whole ? 4 : 1][RT * 4][64], own[whole ? 16 : 1][RT * 16 + 4];
  const bool early = gridDim.y == 1 && row < A.rows;  // else the tile's other workgroups would read the row too
  if (early)
#pragma unroll
    for (int g = 0; g < G; ++g) load(y[g], g);
  const int32_t id = adapter_of(A, row);
  if (blockIdx.y == 0 && id < 0 && row < A.rows && A.out != A.y)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (!early) load(y[g], g);
      store(y[g], g);
    }
  each_adapter(id, blockIdx.y, gridDim.y, [&](int32_t a, bool mine) {
    // everything that the lane reads is on its way before the first product
    const T* w = static_cast<const T*>(A.b) + static_cast<int64_t>(a) * A.d_out * A.rank;
    typename S::V wf[G][2][H::N];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // the channel of row m of the operand: the lane of results 4 j .. 4 j + 3 gets those that are its own
        const int32_t o = o_lo + g * 32 + (H::wide ? u * 16 + n : (n >> 2) * 8 + u * 4 + (n & 3));
#pragma unroll
        for (int c = 0; c < H::N; ++c) {
          const int32_t k = H::entry(c, j, A.rank);
          wf[g][u][c] = typename S::V{};
          if (o < A.d_out && k < A.rank) wf[g][u][c] = *reinterpret_cast<const typename S::V*>(w + static_cast<int64_t>(o) * A.rank + k);
        }
      }
    if (!early && mine)
#pragma unroll
      for (int g = 0; g < G; ++g) load(y[g], g);
    const float* from = A.h + row * A.rank;
    if constexpr (whole) {
      f32x4 acc[RT];
      down_share<T, RT, 4>(A, static_cast<const T*>(A.x) + row * A.x_stride, a, 0, mine, wave, n, j, acc);
      down_join<RT, 4>(red, acc, wave, lane, [&](int k, float sum) { own[n][k] = sum; });
      __syncthreads();
      from = own[n];
    }
    H h;
    h.load(A, from, mine, j);
    const float scale = (A.scale ? A.scale[a] : 1.0f) * h.unit;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      f32x4 acc[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        acc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < H::N; ++c)
#pragma unroll
          for (int p = 0; p < H::pieces; ++p) acc[u] = S::mul(wf[g][u][c], h.v[p][c], acc[u]);
      }
      if (mine) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          z[i] = fmaf(scale, acc[0][i], y[g][i]);
          z[4 + i] = fmaf(scale, acc[1][i], y[g][4 + i]);
        }
        store(z, g);
      }
    }
  });
}

template <typename T, int RT>
hipError_t down(const LoraArgs& A, hipStream_t st) {
  const unsigned tiles = static_cast<unsigned>((A.rows + 15) / 16);
  // few tiles: the adapters of a tile side by side
  const unsigned turns = tiles < 512 ? 16 : 1;
  // and with very few the rank's tiles too, each with its part of A, but x read again for each (rank 64, d_in 2048,
  // bf16, d_out 512: 16 rows 9.6 us, else 15.3; 512 rows of their own adapters 34.7, else 30.4)
  if (RT > 1 && tiles < 16)
    k_lora_down<T, 1><<<dim3(tiles, turns, (A.rank + 15) / 16), 64 * kDownWaves, 0, st>>>(A);
  else
    k_lora_down<T, RT><<<dim3(tiles, turns), 64 * kDownWaves, 0, st>>>(A);
  return hipGetLastError();
}

template <typename T, int RT, bool whole>
hipError_t up(const LoraArgs& A, hipStream_t st) {
  const unsigned tiles = static_cast<unsigned>((A.rows + 15) / 16);
  const unsigned chunks = static_cast<unsigned>((A.d_out + kUpChannels - 1) / kUpChannels);
  const unsigned turns = static_cast<int64_t>(tiles) * chunks < 512 ? 16 : 1;
  k_lora_up<T, RT, whole><<<dim3(tiles * chunks, turns), 256, 0, st>>>(A);
  return hipGetLastError();
}

// f of `most` rows at a time
template <typename T, typename F>
hipError_t each_part(const LoraArgs& A, int64_t most, F&& f) {
  for (int64_t row0 = 0; row0 < A.rows; row0 += most) {
    LoraArgs B = A;
    B.rows = static_cast<int32_t>(A.rows - row0 < most ? A.rows - row0 : most);
    B.x = static_cast<const T*>(A.x) + row0 * A.x_stride;
    B.y = static_cast<const T*>(A.y) + row0 * A.y_stride;
    B.out = static_cast<T*>(A.out) + row0 * A.out_stride;
    B.adapter = A.adapter + row0;
    B.h = A.h + row0 * A.rank;
    const hipError_t e = f(B);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// A launch has fewer than 2^32 threads: more rows are taken a part at a time, all of x
// read before the first of out is written, which may overlap it.
template <typename T, int RT>
hipError_t run(const LoraArgs& A, hipStream_t st) {
  if constexpr (RT <= 2)
    if (A.whole) return up<T, RT, true>(A, st);
  const int64_t chunks = (A.d_out + kUpChannels - 1) / kUpChannels;
  constexpr int64_t threads = (int64_t{1} << 32) - 1;
  const hipError_t e = each_part<T>(A, 16 * (threads / (64 * kDownWaves)), [&](const LoraArgs& B) { return down<T, RT>(B, st); });
  if (e != hipSuccess) return e;
  return each_part<T>(A, 16 * (threads / (256 * chunks)), [&](const LoraArgs& B) { return up<T, RT, false>(B, st); });
}

template <typename T>
hipError_t by_rank(const LoraArgs& A, hipStream_t st) {
  return A.rank <= 16 ? run<T, 1>(A, st) : A.rank <= 32 ? run<T, 2>(A, st) : A.rank <= 64 ? run<T, 4>(A, st) : run<T, 8>(A, st);
}

}  // namespace

// Few rows and a small A: one launch, with h computed once for each 256 channels of
// d_out.  8 rows of their own adapters, 256 -> 768, rank 16: 3.9 us in bf16 and 4.5 in
// fp32, in two launches 6.0 and 6.9; 256 rows, 1024 -> 1024: 9.9 and 17, in two 9.2 and 11.
bool lora_whole(int64_t rows, int32_t d_in, int32_t d_out, int32_t rank) {
  return rows <= 256 && rank <= 32 && d_out <= 4 * kUpChannels && static_cast<int64_t>(d_in) * rank <= 16384 &&
         rows * d_in * rank <= (1 << 20);
}

hipError_t launch_lora(const LoraArgs& A, int dtype, hipStream_t st) {
  return dtype == LB_F32 ? by_rank<float>(A, st) : dtype == LB_BF16 ? by_rank<__bf16>(A, st) : by_rank<_Float16>(A, st);
}

}  // namespace lb
