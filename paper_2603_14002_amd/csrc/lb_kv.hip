// The paged 4-bit cache: append with rotation, read back, and attention.
//
// A block of 32 channels is held as e2m1 codes under a power of two, so a code
// times its scale is exact in bf16 and the matrix instructions take the cache's
// values without a rounding.  gfx950 converts codes to bf16 with the scale in
// one instruction per two values (cvt_scalef32_pk_bf16_fp4), whose scale operand
// is 2^(byte - 127) for the float bits byte << 23, and NaN for byte 255.
#include <hip/hip_runtime.h>

#include "lb_scorer.h"

namespace lb {
namespace {

constexpr int kPoison = 255;  // scale byte of a block with an infinity or a NaN

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ void raise(uint32_t* flags, uint32_t bit) {
  if (flags) atomicOr(flags, bit);
}

// A sequence's rows and tokens, made safe: rows inside 0..n_rows, a length
// inside the page table, at most max_new new tokens, none before position 0.
struct Seq {
  int32_t row0, count, pos0, len;
  bool bad;
};
__device__ __forceinline__ Seq sequence(const KvArgs& A, int32_t s) {
  Seq q;
  const int32_t a = A.starts[s], z = A.starts[s + 1], len = A.lengths[s];
  const int64_t room = static_cast<int64_t>(A.max_pages) << A.page_shift;
  const int32_t most = room < 0x7FFFFFFF ? static_cast<int32_t>(room) : 0x7FFFFFFF;
  q.len = min(max(len, 0), most);
  q.row0 = min(max(a, 0), A.n_rows);
  const int32_t end = min(max(z, q.row0), A.n_rows);
  q.count = min(end - q.row0, A.max_new);
  q.pos0 = q.len - (end - q.row0);
  q.bad = q.len != len || q.row0 != a || end != z || q.count != end - q.row0 || q.pos0 < 0;
  return q;
}

// The page and slot of a token; page < 0: not in the cache's pages.
__device__ __forceinline__ int64_t page_of(const KvArgs& A, int32_t s, int32_t t) {
  const int32_t p = A.table[static_cast<int64_t>(s) * A.max_pages + (t >> A.page_shift)];
  return (p < 0 || p >= A.n_pages) ? -1 : p;
}

// Units of work of append and read: the aligned groups of four positions that a
// sequence's new tokens touch (four tokens' values lie side by side in the
// cache).  count new tokens touch at most count / 4 + 2 groups, so sequence s
// owns units starts[s] / 4 + 2 s and on; with one new token each, unit s.  The
// sequence of a unit is found by the wavefront in 64-way steps.
__device__ __forceinline__ int32_t unit_sequence(const KvArgs& A, int32_t u, int32_t* group) {
  if (A.max_new == 1) {
    *group = 0;
    return u;
  }
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, n = A.n_seqs;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int32_t step = (n + 63) >> 6;
    const int32_t at = lo + min(lane * step, n - 1);
    const bool below = lane * step < n && static_cast<int64_t>(A.starts[at] >> 2) + 2ll * at <= u;
    const int32_t k = max(1, static_cast<int32_t>(__popcll(__ballot(below)))) - 1;
    n = min(step, n - k * step);
    lo += k * step;
  }
  *group = u - ((A.starts[lo] >> 2) + 2 * lo);
  return lo;
}

__device__ __forceinline__ int32_t quad_max(int32_t x) {
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  return max(x, __builtin_amdgcn_mov_dpp(x, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}

// The exponent of a block's scale, from the ordered bits of its largest
// magnitude (`frac` fraction bits, exponent biased by `bias`): with a = m 2^p,
// 1 <= m < 2, the smallest e with a <= 6 * 2^e = 1.5 * 2^(e+2) is p - 2 for m <=
// 1.5, else p - 1.
template <int frac, int bias>
__device__ __forceinline__ int32_t block_exponent(int32_t am) {
  const int32_t p = (am >> frac) - bias;
  const int32_t e = p - 2 + ((am & ((1 << frac) - 1)) > (1 << (frac - 1)));
  return min(max(e, -124), 125);
}

// Eight scaled magnitudes-with-sign to eight codes, rounded to nearest with ties
// to even and clipped at 6.
__device__ __forceinline__ uint32_t codes8(const float (&y)[8]) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
}

// One lane's eight channels of a key, rotated in 64 bits: products of 24-bit
// numbers are exact there, so each value is rounded once, to 53 bits, and its
// block's codes are those of the exact rotation but for values within 2^-53 of
// a border.  The 64-bit value goes on as its upper word with the lower one as a
// sticky bit, which keeps its order and which side of every border it is on.
__device__ __forceinline__ void key_block(const double (&x)[8], uint32_t& codes, int32_t& scale) {
  int32_t hi[8], am = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    hi[i] = __double2hiint(x[i]) | (__double2loint(x[i]) != 0);
    am = max(am, hi[i] & 0x7FFFFFFF);
  }
  am = quad_max(am);
  const int32_t e = block_exponent<20, 1023>(am);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // x / 2^e as a float: 20 fraction bits and the sticky bit; below 2^-126 zero, from 16 on clipped anyway
    const int32_t a = min((hi[i] & 0x7FFFFFFF) - (e << 20), (1023 + 4) << 20);
    const uint32_t m = a >= (897 << 20) ? static_cast<uint32_t>(a - (896 << 20)) << 3 : 0u;
    y[i] = __uint_as_float(m | (static_cast<uint32_t>(hi[i]) & 0x80000000u));
  }
  codes = codes8(y);
  scale = e + 127;
  if (am >= 0x7FF00000) codes = 0, scale = kPoison;
}

// One lane's eight channels of a value: exact in 32 bits as they come.
__device__ __forceinline__ void value_block(const float (&x)[8], uint32_t& codes, int32_t& scale) {
  int32_t am = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) am = max(am, static_cast<int32_t>(__float_as_uint(x[i]) & 0x7FFFFFFFu));
  am = quad_max(am);
  const int32_t e = block_exponent<23, 127>(am);
  const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);  // 2^-e: exact products
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
  codes = codes8(y);
  scale = e + 127;
  if (am >= 0x7F800000) codes = 0, scale = kPoison;
}

// Bytes i of four words as one word (a 4 x 4 byte transpose's row).
__device__ __forceinline__ uint32_t bytes_at(const uint32_t (&w)[4], int i) {
  return (w[0] >> (8 * i) & 255u) | (w[1] >> (8 * i) & 255u) << 8 | (w[2] >> (8 * i) & 255u) << 16 |
         (w[3] >> (8 * i) & 255u) << 24;
}

// A workgroup takes a unit (four positions of a sequence) and 256 of its (head,
// eight channels) items: queries, then keys, then values.  A lane has its
// channels of all four tokens in flight, and the four lanes of a block of 32
// channels agree on the scale by two quad moves.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_append(AppendArgs A) {
  int32_t group;
  const int32_t s = unit_sequence(A.kv, blockIdx.x, &group);
  const Seq q = sequence(A.kv, s);
  if (q.bad && group == 0 && blockIdx.y == 0 && threadIdx.x == 0) raise(A.kv.flags, LB_KV_BAD_LENGTH);
  const int32_t first = max(q.pos0, 0), last = min(q.pos0 + q.count, q.len);  // positions appended: [first, last)
  const int32_t p4 = ((q.pos0 >> 2) + group) << 2;
  if (group < 0 || group > (q.count >> 2) + 1 || p4 >= last || p4 + 4 <= first) return;
  constexpr int C = D / 8;
  const int32_t item = blockIdx.y * 256 + threadIdx.x;
  const int32_t heads = A.kv.q_heads + 2 * A.kv.kv_heads;
  const bool live_item = item < heads * C;
  const int32_t head = live_item ? item / C : heads - 1;  // lanes past the end follow a head, and store nothing
  const int32_t c = item % C, ch = c * 8;
  const int kind = head < A.kv.q_heads ? 0 : head < A.kv.q_heads + A.kv.kv_heads ? 1 : 2;
  bool live[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int32_t p = p4 + t;
    live[t] = p >= first && p < last;
    if (A.rot && live[t] && p >= A.positions) {
      live[t] = false;
      if (item == 0) raise(A.kv.flags, LB_KV_BAD_LENGTH);
    }
  }
  if (!(live[0] || live[1] || live[2] || live[3])) return;
  const int64_t row = q.row0 + (p4 - q.pos0);  // row of the unit's first position (not a live one, perhaps)
  const bool turned = ch < A.rot;
  const int32_t half = A.rot >> 1;

  if (kind == 0) {
    const T* src = static_cast<const T*>(A.q) + head * D;
    T* dst = static_cast<T*>(A.q_out) + head * D;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (!live[t] || !live_item) continue;
      const T* x0 = src + (row + t) * A.q_stride;
      float x[8], r[8];
      load8(x0 + ch, x);
      if (!turned) {
        store8(dst + (row + t) * A.q_out_stride + ch, x);
        continue;
      }
      const int64_t angles = static_cast<int64_t>(p4 + t) * half;
      if (A.interleaved) {
        const f32x4 cs = *reinterpret_cast<const f32x4*>(A.cos + angles + ch / 2);
        const f32x4 sn = *reinterpret_cast<const f32x4*>(A.sin + angles + ch / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          r[2 * i] = fmaf(x[2 * i], cs[i], -(x[2 * i + 1] * sn[i]));
          r[2 * i + 1] = fmaf(x[2 * i + 1], cs[i], x[2 * i] * sn[i]);
        }
        store8(dst + (row + t) * A.q_out_stride + ch, r);
      } else if (ch < half) {
        // a lane turns both halves of its pairs: q_out may be q
        float y[8], cs[8], sn[8], w[8];
        load8(x0 + ch + half, y);
        load8(A.cos + angles + ch, cs);
        load8(A.sin + angles + ch, sn);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          r[i] = fmaf(x[i], cs[i], -(y[i] * sn[i]));
          w[i] = fmaf(y[i], cs[i], x[i] * sn[i]);
        }
        store8(dst + (row + t) * A.q_out_stride + ch, r);
        store8(dst + (row + t) * A.q_out_stride + ch + half, w);
      }
    }
    return;
  }

  const int32_t h = head - A.kv.q_heads - (kind == 2 ? A.kv.kv_heads : 0);
  const int32_t P = 1 << A.kv.page_shift;
  const int64_t page = page_of(A.kv, s, p4);
  if (page < 0) {
    if (c == 0) raise(A.kv.flags, LB_KV_BAD_PAGE);
    return;
  }
  uint8_t* block = A.kv.pages + (page * A.kv.kv_heads + h) * (static_cast<int64_t>(P) * (D + D / 16));
  const int32_t slot = p4 & (P - 1);
  uint32_t codes[4] = {0, 0, 0, 0};
  int32_t scale[4] = {0, 0, 0, 0};
  if (kind == 1) {
    const T* src = static_cast<const T*>(A.k) + h * D;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      double r[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (live[t]) {
        const T* x0 = src + (row + t) * A.k_stride;
        float x[8];
        load8(x0 + ch, x);
        const int64_t angles = static_cast<int64_t>(p4 + t) * half;
        if (!turned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) r[i] = x[i];
        } else if (A.interleaved) {
          const f32x4 cs = *reinterpret_cast<const f32x4*>(A.cos + angles + ch / 2);
          const f32x4 sn = *reinterpret_cast<const f32x4*>(A.sin + angles + ch / 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const double a = x[2 * i], b = x[2 * i + 1], c0 = cs[i], s0 = sn[i];
            r[2 * i] = fma(a, c0, -(b * s0));
            r[2 * i + 1] = fma(b, c0, a * s0);
          }
        } else {
          float y[8], cs[8], sn[8];
          const bool low = ch < half;
          load8(x0 + (low ? ch + half : ch - half), y);
          load8(A.cos + angles + (low ? ch : ch - half), cs);
          load8(A.sin + angles + (low ? ch : ch - half), sn);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double b = static_cast<double>(y[i]) * static_cast<double>(sn[i]);
            r[i] = fma(static_cast<double>(x[i]), static_cast<double>(cs[i]), low ? -b : b);
          }
        }
      }
      key_block(r, codes[t], scale[t]);
    }
    if (!live_item) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (!live[t]) continue;
      *reinterpret_cast<uint32_t*>(block + (slot + t) * (D / 2) + c * 4) = codes[t];
      if ((c & 3) == 0) block[P * D + (slot + t) * (D / 32) + (c >> 2)] = static_cast<uint8_t>(scale[t]);
    }
    return;
  }
  const T* src = static_cast<const T*>(A.v) + h * D;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (live[t]) load8(src + (row + t) * A.v_stride + ch, x);
    value_block(x, codes[t], scale[t]);
  }
  if (!live_item) return;
  uint8_t* at = block + P * D / 2 + ((slot >> 2) * (D / 2) + c * 4) * 4;
  uint8_t* scale_at = block + P * D + P * D / 32 + ((slot >> 2) * (D / 32) + (c >> 2)) * 4;
  if (live[0] && live[1] && live[2] && live[3]) {
    *reinterpret_cast<u32x4*>(at) = u32x4{bytes_at(codes, 0), bytes_at(codes, 1), bytes_at(codes, 2), bytes_at(codes, 3)};
    if ((c & 3) == 0)
      *reinterpret_cast<uint32_t*>(scale_at) = static_cast<uint32_t>(scale[0]) | static_cast<uint32_t>(scale[1]) << 8 |
                                               static_cast<uint32_t>(scale[2]) << 16 | static_cast<uint32_t>(scale[3]) << 24;
    return;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (!live[t]) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) at[4 * i + t] = static_cast<uint8_t>(codes[t] >> (8 * i));
    if ((c & 3) == 0) scale_at[t] = static_cast<uint8_t>(scale[t]);
  }
}

__device__ __forceinline__ void values8(uint32_t codes, uint32_t byte, float (&x)[8]) {
  const float s = scale_of(byte);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1),
              c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
}

template <int D, typename T>
__global__ __launch_bounds__(256) void k_read(ReadArgs A) {
  int32_t group;
  const int32_t s = unit_sequence(A.kv, blockIdx.x, &group);
  const Seq q = sequence(A.kv, s);
  if (q.bad && group == 0 && blockIdx.y == 0 && threadIdx.x == 0) raise(A.kv.flags, LB_KV_BAD_LENGTH);
  const int32_t first = max(q.pos0, 0), last = min(q.pos0 + q.count, q.len);
  const int32_t p4 = ((q.pos0 >> 2) + group) << 2;
  if (group < 0 || group > (q.count >> 2) + 1 || p4 >= last || p4 + 4 <= first) return;
  constexpr int C = D / 8;
  const int32_t item = blockIdx.y * 256 + threadIdx.x;
  if (item >= 2 * A.kv.kv_heads * C) return;
  const int32_t head = item / C, c = item % C;
  const bool key = head < A.kv.kv_heads;
  T* dst = static_cast<T*>(key ? A.k : A.v);
  if (!dst) return;
  const int32_t h = key ? head : head - A.kv.kv_heads;
  const int64_t stride = key ? A.k_stride : A.v_stride;
  const int32_t P = 1 << A.kv.page_shift;
  const int64_t page = page_of(A.kv, s, p4);
  if (page < 0) {
    if (c == 0) raise(A.kv.flags, LB_KV_BAD_PAGE);
    return;
  }
  const uint8_t* block = A.kv.pages + (page * A.kv.kv_heads + h) * (static_cast<int64_t>(P) * (D + D / 16));
  const int32_t slot = p4 & (P - 1);
  uint32_t codes[4], scales;
  if (key) {
    scales = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      codes[t] = *reinterpret_cast<const uint32_t*>(block + (slot + t) * (D / 2) + c * 4);
      scales |= static_cast<uint32_t>(block[P * D + (slot + t) * (D / 32) + (c >> 2)]) << (8 * t);
    }
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4*>(block + P * D / 2 + ((slot >> 2) * (D / 2) + c * 4) * 4);
    const uint32_t in[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
    for (int t = 0; t < 4; ++t) codes[t] = bytes_at(in, t);
    scales = *reinterpret_cast<const uint32_t*>(block + P * D + P * D / 32 + ((slot >> 2) * (D / 32) + (c >> 2)) * 4);
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (p4 + t < first || p4 + t >= last) continue;
    float x[8];
    values8(codes[t], scales >> (8 * t) & 255u, x);
    store8(dst + (q.row0 + (p4 + t - q.pos0)) * stride + h * D + c * 8, x);
  }
}

// ------------------------------------------------------------------ attention
//
// One wavefront multiplies 32 tokens' keys with 16 query rows (a row: a new
// token and one of the query heads that share the KV head) and the
// probabilities with the tokens' values, all by 16x16x32 matrix instructions on
// transposed operands: S^T = K Q^T and O^T = V^T P^T.  An operand's lane (n =
// lane % 16, j = lane / 16) holds 8 entries of its row or column n; a result's
// lane holds column n and rows 4 j .. 4 j + 3.  So
//   - the scores that a lane gets are of its query row n and the tokens 4 j + i
//     of both halves of the tile, which are the 8 entries that it has to hold of
//     P^T: the probabilities never leave their lane;
//   - which channels an instruction takes together is free as long as both
//     operands agree: lane (n, j) takes a contiguous quarter of token n's key,
//     one load, and the values' channels D/16 n .. D/16 (n + 1) - 1 of four
//     adjacent tokens, one load of D/32 words, converted with one scale per
//     token and regrouped by byte permutes.
// A row's maximum is shared by its four lanes after each tile; sums stay in the
// lanes until the end.
//
// Scores, maxima, sums and outputs are held in 32 bits.  The matrix operands are
// bf16: keys and values exactly; queries and probabilities in `NP` pieces, each
// the rounding of what the ones before leave: one piece (relative error 2^-9 of a
// probability) for bf16, whose output has that rounding anyway, two (2^-17) for
// fp16, three (2^-25) for fp32.  bf16 queries are exact with one, fp16 ones with two.

template <typename T>
struct Pieces;
template <>
struct Pieces<__bf16> {
  static constexpr int n = 1;
};
template <>
struct Pieces<_Float16> {
  static constexpr int n = 2;
};
template <>
struct Pieces<float> {
  static constexpr int n = 3;
};

template <int NP>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&w)[NP]) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int k = 0; k < NP; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[k][i] = static_cast<__bf16>(rest[i]);
      // an infinity is one piece: the rest of it would be NaN
      if (k + 1 < NP) rest[i] = __builtin_isinf(rest[i]) ? 0.0f : rest[i] - static_cast<float>(w[k][i]);
    }
}

__device__ __forceinline__ bf16x8 eight(bf16x2 a, bf16x2 b, bf16x2 c, bf16x2 d) {
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

__device__ __forceinline__ bf16x8 bf16_of(uint32_t codes, float s) {
  return eight(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1),
               __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
}

// the maximum (sum) over the four lanes of a query row
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// One half (16 tokens) of a tile in the cache's form.
template <int D>
struct Half {
  uint32_t k[D / 32];  // D/4 codes: the lane's quarter of key n
  uint32_t v[D / 32];  // values of tokens 4 j .. 4 j + 3, channel pairs D/32 n .. D/32 (n + 1) - 1
  uint32_t ks;         // scale bytes of the quarter's blocks (one, or two with D = 256)
  uint32_t vs;         // scale bytes of the four tokens' values
  bool ok;             // the page exists
};

template <int D>
__device__ __forceinline__ void load_half(const KvArgs& A, int32_t s, int32_t h, int32_t t0, int32_t end, int n, int j, Half<D>& H) {
  const int64_t page = t0 < end ? page_of(A, s, t0) : -2;
  H.ok = page >= 0;
  if (!H.ok) {
    if (page == -1) raise(A.flags, LB_KV_BAD_PAGE);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) H.k[i] = H.v[i] = 0;
    H.ks = H.vs = 0;
    return;
  }
  const int32_t P = 1 << A.page_shift, slot = t0 & (P - 1);
  const uint8_t* block = A.pages + (page * A.kv_heads + h) * (static_cast<int64_t>(P) * (D + D / 16));
  const uint8_t* k = block + (slot + n) * (D / 2) + j * (D / 8);
  const uint8_t* v = block + P * D / 2 + (((slot >> 2) + j) * (D / 2) + n * (D / 32)) * 4;
  if constexpr (D == 64) {
    const u32x2 a = *reinterpret_cast<const u32x2*>(k), b = *reinterpret_cast<const u32x2*>(v);
    H.k[0] = a.x, H.k[1] = a.y, H.v[0] = b.x, H.v[1] = b.y;
  } else {
#pragma unroll
    for (int i = 0; i < D / 128; ++i) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(k + 16 * i), b = *reinterpret_cast<const u32x4*>(v + 16 * i);
#pragma unroll
      for (int x = 0; x < 4; ++x) H.k[4 * i + x] = a[x], H.v[4 * i + x] = b[x];
    }
  }
  const uint8_t* ks = block + P * D + (slot + n) * (D / 32) + (j * D) / 128;
  H.ks = D == 256 ? *reinterpret_cast<const uint16_t*>(ks) : *ks;
  H.vs = *reinterpret_cast<const uint32_t*>(block + P * D + P * D / 32 + (((slot >> 2) + j) * (D / 32) + (n * D) / 512) * 4);
}

__device__ __forceinline__ bool any_poison(uint32_t w) {
  return ((w & 0xFFu) == 0xFFu) || ((w & 0xFF00u) == 0xFF00u) || ((w & 0xFF0000u) == 0xFF0000u) || (w >> 24) == 0xFFu;
}

// A workgroup takes 16 query rows of one sequence and KV head and one part of
// their key range; its four wavefronts take every fourth tile and join at the end.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_attend(AttendArgs A) {
  constexpr int NP = Pieces<T>::n, KC = D / 32, VC = D / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, j = lane >> 4;
  const int32_t split = blockIdx.x % A.splits;
  int64_t rest = blockIdx.x / A.splits;
  const int32_t h = static_cast<int32_t>(rest % A.kv.kv_heads);
  rest /= A.kv.kv_heads;
  const int32_t tile = static_cast<int32_t>(rest % A.tiles), s = static_cast<int32_t>(rest / A.tiles);
  const Seq q = sequence(A.kv, s);
  if (q.bad && tile == 0 && h == 0 && split == 0 && threadIdx.x == 0) raise(A.kv.flags, LB_KV_BAD_LENGTH);
  const int32_t G = A.kv.q_heads / A.kv.kv_heads;
  const int32_t R = q.count * G, r0 = tile * 16;
  if (r0 >= R) return;
  const bool live = r0 + n < R;
  const int32_t i_tok = (r0 + n) / G, g = (r0 + n) % G;
  const int32_t pos = live ? q.pos0 + i_tok : -1;
  const int64_t row = q.row0 + static_cast<int64_t>(i_tok);
  const int32_t hq = h * G + g;

  // keys that some row of the tile sees, and this part of them
  const int32_t p_first = q.pos0 + r0 / G;
  const int32_t p_last = q.pos0 + (min(R, r0 + 16) - 1) / G;
  const int32_t end = min(q.len, p_last + 1);
  const int32_t begin = A.window > 0 ? max(0, p_first - A.window + 1) & ~31 : 0;
  const int32_t tiles = end > begin ? (end - begin + 31) >> 5 : 0;
  const int32_t per = (tiles + A.splits - 1) / A.splits;
  const int32_t t_lo = split * per, t_hi = min(tiles, t_lo + per);

  bf16x8 qf[KC][NP];
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (live) load8(static_cast<const T*>(A.q) + row * A.q_stride + hq * D + j * (D / 4) + c * 8, x);
    split8<NP>(x, qf[c]);
  }

  f32x4 o[VC];
#pragma unroll
  for (int c = 0; c < VC; ++c) o[c] = f32x4{0, 0, 0, 0};
  float m = -__builtin_inff(), l = 0.0f;

  for (int32_t t = t_lo + wave; t < t_hi; t += 4) {
    const int32_t tb = begin + t * 32;
    Half<D> H[2];
    load_half<D>(A.kv, s, h, tb, end, n, j, H[0]);
    load_half<D>(A.kv, s, h, tb + 16, end, n, j, H[1]);
    float sc[8];
    bool seen[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 acc{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        // channels j D/4 + 8 c .. + 7 lie in block (8 c) / 32 of the quarter (D = 256 has two there)
        const uint32_t byte = D == 256 ? (H[u].ks >> (c < KC / 2 ? 0 : 8)) & 255u : H[u].ks;
        const bf16x8 kf = bf16_of(H[u].k[c], scale_of(byte));
#pragma unroll
        for (int p = 0; p < NP; ++p) acc = mfma(kf, qf[c][p], acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t tok = tb + 16 * u + 4 * j + i;
        const bool vis = H[u].ok && tok < end && tok <= pos && (A.window <= 0 || tok > pos - A.window);
        seen[4 * u + i] = vis;
        sc[4 * u + i] = vis ? acc[i] * A.scale2 : -__builtin_inff();
      }
    }
    float mx = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, sc[i]);
    mx = row_max(mx);
    const float base = mx == -__builtin_inff() ? 0.0f : mx;  // nothing seen yet: every exponent is -infinity
    const float fade = __builtin_amdgcn_exp2f(m - base);
    m = mx;
    l *= fade;
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(sc[i] - base);
      l += p[i];
    }
#pragma unroll
    for (int c = 0; c < VC; ++c) o[c] *= fade;
    bf16x8 pf[NP];
    split8<NP>(p, pf);

    // the values' scales; tokens that no row sees count as 0, whatever the cache holds there
    float vs[2][4];
    bool poison = false;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t byte = H[u].vs >> (8 * i) & 255u;
        const bool in = tb + 16 * u + 4 * j + i < end;
        poison |= in && byte == kPoison;
        vs[u][i] = scale_of(in && byte != kPoison ? byte : 0u);
      }
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      uint32_t y[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        y[u][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(H[u].v[w], vs[u][0], 0));
        y[u][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(H[u].v[w], vs[u][1], 1));
        y[u][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(H[u].v[w], vs[u][2], 2));
        y[u][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(H[u].v[w], vs[u][3], 3));
      }
#pragma unroll
      for (int par = 0; par < 2; ++par) {
        // the even (odd) channel of the pair for the eight tokens
        const uint32_t sel = par ? 0x07060302u : 0x05040100u;
        const u32x4 f{__builtin_amdgcn_perm(y[0][1], y[0][0], sel), __builtin_amdgcn_perm(y[0][3], y[0][2], sel),
                      __builtin_amdgcn_perm(y[1][1], y[1][0], sel), __builtin_amdgcn_perm(y[1][3], y[1][2], sel)};
        const bf16x8 vf = __builtin_bit_cast(bf16x8, f);
#pragma unroll
        for (int k = 0; k < NP; ++k) o[2 * w + par] = mfma(vf, pf[k], o[2 * w + par]);
      }
    }
    if (__any(poison)) {
      // a block of NaN reaches the rows that see its token, and no other: 0 * NaN
      // in the products above would reach all of them
      bf16x8 bad, vis;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool b = (H[i >> 2].vs >> (8 * (i & 3)) & 255u) == kPoison && tb + 16 * (i >> 2) + 4 * j + (i & 3) < end;
        bad[i] = static_cast<__bf16>(b ? 1.0f : 0.0f);
        vis[i] = static_cast<__bf16>(seen[i] ? 1.0f : 0.0f);
      }
      const f32x4 hit = mfma(bad, vis, f32x4{0, 0, 0, 0});
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (hit[i] > 0.0f)
#pragma unroll
          for (int c = 0; c < VC; ++c) o[c][i] = __builtin_nanf("");
    }
  }
  l = row_sum(l);

  // join the four wavefronts
  __shared__ float part[4][VC * 4][64];
  __shared__ float pm[4][16], pl[4][16];
#pragma unroll
  for (int c = 0; c < VC; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][4 * c + i][lane] = o[c][i];
  if (j == 0) pm[wave][n] = m, pl[wave][n] = l;
  __syncthreads();
  const float M = fmaxf(fmaxf(pm[0][n], pm[1][n]), fmaxf(pm[2][n], pm[3][n]));
  const float base = M == -__builtin_inff() ? 0.0f : M;
  float wgt[4], L = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    wgt[w] = __builtin_amdgcn_exp2f(pm[w][n] - base);
    L += wgt[w] * pl[w][n];
  }
  if (!live) return;
  // wave w writes the rows 4 j + w of the results: D/16 adjacent channels a lane
  const int i = wave;
  float x[VC];
#pragma unroll
  for (int c = 0; c < VC; ++c) {
    x[c] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) x[c] += wgt[w] * part[w][4 * c + i][lane];
  }
  const int32_t ch = (4 * j + i) * (D / 16);
  if (A.splits > 1) {
    const int64_t slot = (row * A.kv.q_heads + hq) * A.splits + split;
    float* dst = A.part + slot * (D + 2);
    if (i == 0 && j == 0) dst[D] = M, dst[D + 1] = L;
#pragma unroll
    for (int c = 0; c < VC; ++c) dst[ch + c] = x[c];
    return;
  }
  const float inv = L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : L;  // L may be NaN
  T* dst = static_cast<T*>(A.out) + row * A.out_stride + hq * D + ch;
#pragma unroll
  for (int c = 0; c < VC; ++c) dst[c] = static_cast<T>(x[c] * inv);
  if (A.lse && i == 0 && j == 0)
    A.lse[row * A.kv.q_heads + hq] = L == 0.0f ? -__builtin_inff() : (base + log2f(L)) * 0.6931471805599453f;
}

// Joins the parts of a row's key range: a wavefront per (new token, query head).
template <int D, typename T>
__global__ __launch_bounds__(64) void k_attend_join(AttendArgs A) {
  const int32_t hq = blockIdx.y;
  const int64_t row = blockIdx.x;
  if (row < A.kv.starts[0] || row >= A.kv.starts[A.kv.n_seqs]) return;  // padding
  const int lane = threadIdx.x;
  const float* src = A.part + (row * A.kv.q_heads + hq) * A.splits * (D + 2);
  float M = -__builtin_inff();
  for (int32_t k = 0; k < A.splits; ++k) M = fmaxf(M, src[k * (D + 2) + D]);
  const float base = M == -__builtin_inff() ? 0.0f : M;
  float L = 0.0f, x[D / 64];
#pragma unroll
  for (int c = 0; c < D / 64; ++c) x[c] = 0.0f;
  for (int32_t k = 0; k < A.splits; ++k) {
    const float* p = src + k * (D + 2);
    const float w = __builtin_amdgcn_exp2f(p[D] - base);
    L += w * p[D + 1];
#pragma unroll
    for (int c = 0; c < D / 64; ++c) x[c] += w * p[c * 64 + lane];
  }
  const float inv = L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : L;
  T* dst = static_cast<T*>(A.out) + row * A.out_stride + hq * D;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) dst[c * 64 + lane] = static_cast<T>(x[c] * inv);
  if (A.lse && lane == 0)
    A.lse[row * A.kv.q_heads + hq] = L == 0.0f ? -__builtin_inff() : (base + log2f(L)) * 0.6931471805599453f;
}

int64_t units(const KvArgs& A) { return A.max_new == 1 ? A.n_seqs : A.n_rows / 4 + 2ll * A.n_seqs; }

template <int D, typename T>
hipError_t append(const AppendArgs& A, hipStream_t st) {
  const int64_t items = (A.kv.q_heads + 2ll * A.kv.kv_heads) * (D / 8);
  k_append<D, T><<<dim3(static_cast<unsigned>(units(A.kv)), static_cast<unsigned>((items + 255) / 256)), 256, 0, st>>>(A);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t read(const ReadArgs& A, hipStream_t st) {
  const int64_t items = 2ll * A.kv.kv_heads * (D / 8);
  k_read<D, T><<<dim3(static_cast<unsigned>(units(A.kv)), static_cast<unsigned>((items + 255) / 256)), 256, 0, st>>>(A);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t attend(const AttendArgs& A, hipStream_t st) {
  const int64_t blocks = static_cast<int64_t>(A.kv.n_seqs) * A.tiles * A.kv.kv_heads * A.splits;
  k_attend<D, T><<<dim3(static_cast<unsigned>(blocks)), 256, 0, st>>>(A);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.splits == 1) return e;
  k_attend_join<D, T><<<dim3(static_cast<unsigned>(A.kv.n_rows), static_cast<unsigned>(A.kv.q_heads)), 64, 0, st>>>(A);
  return hipGetLastError();
}

}  // namespace

#define LB_KV_DISPATCH(fn)                                                        \
  do {                                                                            \
    if (head_dim == 64)                                                           \
      return dtype == LB_F32 ? fn<64, float>(A, st) : dtype == LB_BF16 ? fn<64, __bf16>(A, st) : fn<64, _Float16>(A, st); \
    if (head_dim == 128)                                                          \
      return dtype == LB_F32 ? fn<128, float>(A, st) : dtype == LB_BF16 ? fn<128, __bf16>(A, st) : fn<128, _Float16>(A, st); \
    return dtype == LB_F32 ? fn<256, float>(A, st) : dtype == LB_BF16 ? fn<256, __bf16>(A, st) : fn<256, _Float16>(A, st); \
  } while (0)

hipError_t launch_kv_append(const AppendArgs& A, int head_dim, int dtype, hipStream_t st) { LB_KV_DISPATCH(append); }
hipError_t launch_kv_read(const ReadArgs& A, int head_dim, int dtype, hipStream_t st) { LB_KV_DISPATCH(read); }
hipError_t launch_kv_attend(const AttendArgs& A, int head_dim, int dtype, hipStream_t st) { LB_KV_DISPATCH(attend); }

// Tiles of 16 query rows a sequence may have, and the parts of its key range:
// so many that about four workgroups a CU exist, each with 8 tiles of keys at least.
AttendPlan attend_plan(const KvArgs& kv, int head_dim) {
  AttendPlan p;
  const int64_t rows = static_cast<int64_t>(kv.max_new) * (kv.q_heads / kv.kv_heads);
  p.tiles = static_cast<int32_t>((rows + 15) / 16);
  const int64_t blocks = static_cast<int64_t>(kv.n_seqs) * p.tiles * kv.kv_heads;
  const int64_t tokens = static_cast<int64_t>(kv.max_pages) << kv.page_shift;
  int64_t s = blocks > 0 ? (1024 + blocks - 1) / blocks : 1;
  s = s < tokens / 256 ? s : tokens / 256;
  p.splits = static_cast<int32_t>(s < 1 ? 1 : s > 128 ? 128 : s);
  p.part_floats = p.splits > 1 ? static_cast<int64_t>(kv.n_rows) * kv.q_heads * p.splits * (head_dim + 2) : 0;
  return p;
}

}  // namespace lb
