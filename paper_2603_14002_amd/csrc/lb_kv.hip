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

// A sequence whose starts or length do not fit is reported by one workgroup, whichever rows it has itself.
__device__ __forceinline__ void check_sequence(const KvArgs& A, uint32_t s) {
  if (s < static_cast<uint32_t>(A.n_seqs) && threadIdx.x == 0 && sequence(A, static_cast<int32_t>(s)).bad) raise(A.flags, LB_KV_BAD_LENGTH);
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

// The same for tiles of `per` query rows, `group` to a new token: sequence s owns
// units starts[s] * group / per + s and on, and has no more tiles than those.
__device__ __forceinline__ int32_t row_unit(const KvArgs& A, int32_t u, int32_t group, int32_t per, int32_t* tile) {
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, n = A.n_seqs;
  while (n > 1) {
    const int32_t step = (n + 63) >> 6;
    const int32_t at = lo + min(lane * step, n - 1);
    const bool below = lane * step < n && static_cast<int64_t>(A.starts[at]) * group / per + at <= u;
    const int32_t k = max(1, static_cast<int32_t>(__popcll(__ballot(below)))) - 1;
    n = min(step, n - k * step);
    lo += k * step;
  }
  const int64_t t = u - (static_cast<int64_t>(A.starts[lo]) * group / per + lo);
  *tile = t < -1 || t > 0x7FFFFFFF ? -1 : static_cast<int32_t>(t);
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
// channels agree on the scale by two quad moves.  24 000 tokens of 12 prompts, 32 + 16
// heads of 128, bf16: 115 us, 4.5 TB/s; what the rows wait for (starts, lengths, page)
// and the registers of the 64-bit rotation (four wavefronts a SIMD, three in fp32)
// bound it.  Rows are read and written once,
// past the caches (else 128 us).
template <int D, typename T>
__global__ __launch_bounds__(256) void k_append(AppendArgs A) {
  int32_t group;
  const int32_t s = unit_sequence(A.kv, blockIdx.x, &group);
  const Seq q = sequence(A.kv, s);
  if (blockIdx.y == 0) check_sequence(A.kv, blockIdx.x);
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
  // All loads go before the first store, which they would otherwise have to wait
  // for (q_out may be q), and have no branch: a position that is not live takes
  // the data of one that is.
  int32_t pos[4];
  int64_t row[4];
#pragma unroll
  for (int t = 3; t >= 0; --t) {
    pos[t] = p4 + (live[t] ? t : live[0] ? 0 : live[1] ? 1 : live[2] ? 2 : 3);
    row[t] = q.row0 + static_cast<int64_t>(pos[t] - q.pos0);
  }
  const bool turned = ch < A.rot;
  const int32_t half = A.rot >> 1;

  if (kind == 0) {
    const T* src = static_cast<const T*>(A.q) + head * D + ch;
    T* dst = static_cast<T*>(A.q_out) + head * D + ch;
    // a lane turns both halves of its pairs, and the second half's lanes do nothing: q_out may be q
    const bool both = turned && !A.interleaved;
    if (both && ch >= half) return;
    float x[4][8], y[4][8];
#pragma unroll
    for (int t = 0; t < 4; ++t) load8_nt(src + row[t] * A.q_stride, x[t]);
    if (both) {
#pragma unroll
      for (int t = 0; t < 4; ++t) load8_nt(src + row[t] * A.q_stride + half, y[t]);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float cs[8], sn[8];
        load8(A.cos + static_cast<int64_t>(pos[t]) * half + ch, cs);
        load8(A.sin + static_cast<int64_t>(pos[t]) * half + ch, sn);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float a = x[t][i], b = y[t][i];
          x[t][i] = fmaf(a, cs[i], -(b * sn[i]));
          y[t][i] = fmaf(b, cs[i], a * sn[i]);
        }
      }
    } else if (turned) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4 cs = *reinterpret_cast<const f32x4*>(A.cos + static_cast<int64_t>(pos[t]) * half + ch / 2);
        const f32x4 sn = *reinterpret_cast<const f32x4*>(A.sin + static_cast<int64_t>(pos[t]) * half + ch / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = x[t][2 * i], b = x[t][2 * i + 1];
          x[t][2 * i] = fmaf(a, cs[i], -(b * sn[i]));
          x[t][2 * i + 1] = fmaf(b, cs[i], a * sn[i]);
        }
      }
    }
    if (!live_item) return;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (live[t]) {
        store8_nt(dst + row[t] * A.q_out_stride, x[t]);
        if (both) store8_nt(dst + row[t] * A.q_out_stride + half, y[t]);
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
  uint32_t codes[4];
  int32_t scale[4];
  if (kind == 1) {
    const T* src = static_cast<const T*>(A.k) + h * D + ch;
    float x[4][8];
#pragma unroll
    for (int t = 0; t < 4; ++t) load8_nt(src + row[t] * A.k_stride, x[t]);
    if ((ch & ~31) >= A.rot) {  // the whole block stays: the four lanes of a block go the same way
#pragma unroll
      for (int t = 0; t < 4; ++t) value_block(x[t], codes[t], scale[t]);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        double r[8];
        const int64_t angles = static_cast<int64_t>(pos[t]) * half;
        if (!turned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) r[i] = x[t][i];
        } else if (A.interleaved) {
          const f32x4 cs = *reinterpret_cast<const f32x4*>(A.cos + angles + ch / 2);
          const f32x4 sn = *reinterpret_cast<const f32x4*>(A.sin + angles + ch / 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const double a = x[t][2 * i], b = x[t][2 * i + 1], c0 = cs[i], s0 = sn[i];
            r[2 * i] = fma(a, c0, -(b * s0));
            r[2 * i + 1] = fma(b, c0, a * s0);
          }
        } else {
          float y[8], cs[8], sn[8];
          const bool low = ch < half;
          load8_nt(src + row[t] * A.k_stride + (low ? half : -half), y);
          load8(A.cos + angles + (low ? ch : ch - half), cs);
          load8(A.sin + angles + (low ? ch : ch - half), sn);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double b = static_cast<double>(y[i]) * static_cast<double>(sn[i]);
            r[i] = fma(static_cast<double>(x[t][i]), static_cast<double>(cs[i]), low ? -b : b);
          }
        }
        key_block(r, codes[t], scale[t]);
      }
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
  const T* src = static_cast<const T*>(A.v) + h * D + ch;
  float x[4][8];
#pragma unroll
  for (int t = 0; t < 4; ++t) load8_nt(src + row[t] * A.v_stride, x[t]);
#pragma unroll
  for (int t = 0; t < 4; ++t) value_block(x[t], codes[t], scale[t]);
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

// The same units and items, the other way.  24 000 tokens, 16 heads of 128, bf16: 22
// us, 5.7 TB/s, bound by memory.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_read(ReadArgs A) {
  int32_t group;
  const int32_t s = unit_sequence(A.kv, blockIdx.x, &group);
  const Seq q = sequence(A.kv, s);
  if (blockIdx.y == 0) check_sequence(A.kv, blockIdx.x);
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
// bf16: keys and values exactly; queries and probabilities in pieces, each the
// rounding of what the ones before leave.  Queries are exact: one piece for bf16,
// two for fp16, three for fp32.  Probabilities have two for bf16 and fp16 (off by at
// most 2^-16 of a probability: with one, 2^-8, an output would be off by as much
// again as by its own rounding to bf16) and three for fp32 (2^-24).

template <typename T>
struct Pieces;
template <>
struct Pieces<__bf16> {
  static constexpr int q = 1, p = 2;
};
template <>
struct Pieces<_Float16> {
  static constexpr int q = 2, p = 2;
};
template <>
struct Pieces<float> {
  static constexpr int q = 3, p = 3;
};

// large: some x may be infinite or past bf16's largest number.
template <bool large, int N>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&w)[N]) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[k][i] = large && N > 1 && k == 0 ? first_piece(rest[i]) : static_cast<__bf16>(rest[i]);
      if (k + 1 < N) rest[i] = large && k > 0 && __builtin_isinf(rest[i]) ? 0.0f : rest[i] - static_cast<float>(w[k][i]);
    }
}

__device__ __forceinline__ bf16x8 eight(bf16x2 a, bf16x2 b, bf16x2 c, bf16x2 d) {
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

__device__ __forceinline__ bf16x8 bf16_of(uint32_t codes, float s) {
  return eight(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1),
               __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
}

// the larger of two, of a NaN and a number the number (fmaxf would first quiet
// each operand in an instruction of its own)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, __builtin_inff()); }

// the maximum (sum) over the four lanes of a query row
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The value itself, which the compiler does not know: what is computed from it
// stays behind the branch that it stands behind, and is not done ahead for all.
template <typename I>
__device__ __forceinline__ I behind_branch(I x) {
  asm volatile("" : "+v"(x));
  return x;
}

// bit 7 of each byte that is 255: its low seven bits carry into it, and it is set
__device__ __forceinline__ uint32_t carry_255(uint32_t w) { return (w & 0x7F7F7F7Fu) + 0x01010101u & w & 0x80808080u; }

// The pages of a key range: tiles of 32 tokens from `begin` on, of which a
// wavefront takes every `step`-th.  Lane i holds the pages (of both halves of 16
// tokens) of the i-th of the next 64 tiles, so a tile's address needs no load
// before it.  Halves that end before `first`, which nobody sees, have none.
struct Pages {
  const int32_t* table;
  int32_t n_pages, shift, begin, first, end, step;
  static constexpr int32_t kNothing = -(1 << 29);  // no tile is within 64 steps of it
  int32_t held, page0, page1;

  __device__ __forceinline__ Pages(const KvArgs& A, int32_t s, int32_t first_, int32_t end_, int32_t step_)
      : table(A.table + static_cast<int64_t>(s) * A.max_pages), n_pages(static_cast<int32_t>(A.n_pages)), shift(A.page_shift),
        begin(first_ & ~31), first(first_), end(end_), step(step_), held(kNothing), page0(-1), page1(-1) {}

  // makes lane i hold the pages of tile t + i * step
  __device__ __forceinline__ void hold(int32_t t, uint32_t* flags) {
    const int lane = threadIdx.x & 63;
    held = t;
    const int64_t tok = begin + (static_cast<int64_t>(t) + static_cast<int64_t>(lane) * step) * 32;
    const bool seen0 = tok < end && tok + 16 > first, seen1 = tok + 16 < end && tok + 32 > first;
    page0 = seen0 ? table[tok >> shift] : -1;
    page1 = seen1 ? table[(tok + 16) >> shift] : -1;
    if ((seen0 && (page0 < 0 || page0 >= n_pages)) || (seen1 && (page1 < 0 || page1 >= n_pages))) {
      raise(flags, LB_KV_BAD_PAGE);
      if (page0 >= n_pages) page0 = -1;
      if (page1 >= n_pages) page1 = -1;
    }
    // no load is under way when the branches join: else every tile would wait here for all that are (vmcnt 0)
    __builtin_amdgcn_s_waitcnt(0x0F70);
  }

  // the pages of tile t's halves, -1: none
  __device__ __forceinline__ void of(int32_t t, int32_t (&page)[2], uint32_t* flags) {
    int32_t i = (t - held) / step;
    if (i >= 64 || i < 0) {
      hold(t, flags);
      i = 0;
    }
    page[0] = __builtin_amdgcn_readlane(page0, i);
    page[1] = __builtin_amdgcn_readlane(page1, i);
  }
  __device__ __forceinline__ int32_t slot(int32_t t, int u) const { return (begin + t * 32 + 16 * u) & ((1 << shift) - 1); }
};

template <bool once, typename V>
__device__ __forceinline__ V load_as(const uint8_t* p) {
  const V* at = reinterpret_cast<const V*>(p);
  if constexpr (once) return __builtin_nontemporal_load(at);
  return *at;
}
// N words from memory that is aligned to as many (2 or 4: in one load); once: they are read by nobody else
template <int N, bool once = false>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (N == 1) {
    w[0] = load_as<once, uint32_t>(p);
  } else if constexpr (N == 2) {
    const u32x2 a = load_as<once, u32x2>(p);
    w[0] = a.x, w[1] = a.y;
  } else {
#pragma unroll
    for (int c = 0; c < N; c += 4) {
      const u32x4 a = load_as<once, u32x4>(p + 4 * c);
#pragma unroll
      for (int x = 0; x < 4; ++x) w[c + x] = a[x];
    }
  }
}

// A tile (32 tokens) in the cache's form, by halves of 16 tokens.
template <int D>
struct Tile {
  uint32_t k[2][D / 32];  // D/4 codes: the lane's quarter of key n
  uint32_t v[2][D / 32];  // values of tokens 4 j .. 4 j + 3, channel pairs D/32 n .. D/32 (n + 1) - 1
  uint32_t ks[2];         // scale bytes of the quarter's blocks (one, or two with D = 256)
  uint32_t vs[2];         // scale bytes of the four tokens' values
};

// A wavefront's whole tiles of one KV head.
template <int D>
struct Keys {
  Pages P;
  const uint8_t* base;  // the head's part of page 0
  int64_t page_bytes;
  uint32_t k_at, v_at, ks_at, vs_at;

  __device__ __forceinline__ Keys(const KvArgs& A, int32_t s, int32_t h, int32_t first, int32_t end, int32_t step, int n, int j)
      : P(A, s, first, end, step) {
    const int32_t T = 1 << A.page_shift, block = T * (D + D / 16);
    base = A.pages + static_cast<int64_t>(h) * block;
    page_bytes = static_cast<int64_t>(block) * A.kv_heads;
    k_at = n * (D / 2) + j * (D / 8);
    v_at = T * (D / 2) + j * (D * 2) + n * (D / 8);
    ks_at = T * D + n * (D / 32) + j * D / 128;
    vs_at = T * D + T * (D / 32) + (j * (D / 32) + n * D / 512) * 4;
  }

  // loads tile t; bit u of the result: half u exists
  template <bool once>
  __device__ __forceinline__ int load(int32_t t, Tile<D>& X, uint32_t* flags) {
    int32_t page[2];
    P.of(t, page, flags);
    int ok = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (page[u] < 0) continue;  // what the registers hold stays unseen
      ok |= 1 << u;
      const int32_t slot = P.slot(t, u);
      const uint8_t* at = base + page[u] * page_bytes + slot * (D / 2);
      const uint8_t* scales = base + page[u] * page_bytes + slot * (D / 32);
      load_words<D / 32, once>(at + k_at, X.k[u]);
      load_words<D / 32, once>(at + v_at, X.v[u]);
      X.ks[u] = D == 256 ? *reinterpret_cast<const uint16_t*>(scales + ks_at) : scales[ks_at];
      X.vs[u] = *reinterpret_cast<const uint32_t*>(scales + vs_at);
    }
    return ok;
  }
};

// The scale operand of byte i of a word of scale bytes.  The conversion takes the
// exponent bits of its operand and no others (tried with every byte and code on
// gfx950), so the other bytes need not be cleared.
__device__ __forceinline__ float scale_at(uint32_t word, int i) { return __uint_as_float(i == 3 ? word >> 1 : word << (23 - 8 * i)); }

// The values' scales of a tile; tokens before `first` and from `end` on, and of halves
// that do not exist, get the byte 0, whatever the cache holds there (0 times an infinity
// would be NaN), and so do blocks of NaN: which these are is left in `nan`, 255 a byte.
struct ValueScales {
  uint32_t bytes[2], nan[2];
  bool any_nan;  // in some lane

  __device__ __forceinline__ ValueScales(const uint32_t (&vs)[2], int32_t tb, int32_t first, int32_t end, int ok, int j) {
    bytes[0] = vs[0], bytes[1] = vs[1];
    if (ok != 3 || tb < first || tb + 32 > end) {
      const int32_t at = behind_branch(tb);  // most tiles are whole
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int32_t tok = at + 16 * u + 4 * j, left = ok >> u & 1 ? end - tok : 0, before = first - tok;
        bytes[u] = left >= 4 ? bytes[u] : left <= 0 ? 0u : bytes[u] & ((1u << (8 * left)) - 1u);
        bytes[u] = before <= 0 ? bytes[u] : before >= 4 ? 0u : bytes[u] >> (8 * before) << (8 * before);
      }
    }
    nan[0] = nan[1] = 0;
    any_nan = __any((carry_255(bytes[0]) | carry_255(bytes[1])) != 0);
    if (any_nan) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        nan[u] = (carry_255(behind_branch(bytes[u])) >> 7) * 255u;
        bytes[u] &= ~nan[u];
      }
    }
  }

  // one word of values (a channel pair of four tokens) of each half, as bf16: [half][token] channel pairs
  __device__ __forceinline__ void convert(uint32_t w0, uint32_t w1, uint32_t (&y)[2][4]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t w = u ? w1 : w0;
      y[u][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_at(bytes[u], 0), 0));
      y[u][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_at(bytes[u], 1), 1));
      y[u][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_at(bytes[u], 2), 2));
      y[u][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_at(bytes[u], 3), 3));
    }
  }
};
// the even (odd: 1) channel of the pairs for the eight tokens
__device__ __forceinline__ bf16x8 channel(const uint32_t (&y)[2][4], int odd) {
  const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
  const u32x4 f{__builtin_amdgcn_perm(y[0][1], y[0][0], sel), __builtin_amdgcn_perm(y[0][3], y[0][2], sel),
                __builtin_amdgcn_perm(y[1][1], y[1][0], sel), __builtin_amdgcn_perm(y[1][3], y[1][2], sel)};
  return __builtin_bit_cast(bf16x8, f);
}

// The state of QT tiles of 16 query rows in one wavefront.
template <int D, typename T, int QT>
struct Rows {
  static constexpr int KC = D / 32, VC = D / 16, NQ = Pieces<T>::q, NP = Pieces<T>::p;
  bf16x8 q[QT][KC][NQ];
  f32x4 o[QT][VC];
  float m[QT], l[QT];  // reference and the lane's share of the sum of exp2(score - reference)
  int32_t pos[QT];     // the lane's row's position, -1: no row
  float scale2;        // log2(e) |scale|, its sign is in q
  int32_t window, first, end, p_min, p_max;  // over the rows there are: tokens first .. end - 1 are seen by some

  // How far a score may pass the reference before the reference moves: sums of
  // exp2 keep their precision, and most tiles need no exchange between lanes.
  static constexpr float kSlack = 8.0f;

  // every row sees the whole tile at tb
  __device__ __forceinline__ bool inner(int32_t tb, int ok) const {
    return ok == 3 && tb + 31 <= p_min && tb + 32 <= end && (window <= 0 || tb > p_max - window);
  }

  // Scores of a tile's tokens, before the scale; key(u, c): channels j D/4 + 8 c
  // .. + 7 of the lane's token in half u.
  template <typename Key>
  __device__ __forceinline__ void score(Key&& key, f32x4 (&acc)[QT][2]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int t = 0; t < QT; ++t) acc[t][u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const bf16x8 kf = key(u, c);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int p = 0; p < NQ; ++p) acc[t][u] = mfma(kf, q[t][c][p], acc[t][u]);
      }
    }
  }

  // The tokens' probabilities as matrix operands, and their sums.
  __device__ __forceinline__ void weigh(f32x4 (&acc)[QT][2], int32_t tb, int ok, int j, bf16x8 (&pf)[QT][NP]) {
    if (!inner(tb, ok)) {
      const int32_t at = behind_branch(tb);  // most tiles are whole
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          int32_t lo, hi;
          range(t, at + 16 * u + 4 * j, ok >> u & 1, lo, hi);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < lo || i > hi) acc[t][u][i] = -__builtin_inff();
        }
    }
    float top[QT];
    bool past = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      top[t] = scale2 * larger(larger(larger(acc[t][0][0], acc[t][0][1]), larger(acc[t][0][2], acc[t][0][3])),
                               larger(larger(acc[t][1][0], acc[t][1][1]), larger(acc[t][1][2], acc[t][1][3])));
      past |= top[t] > m[t] + kSlack;
    }
    if (__any(past)) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float mx = fmaxf(m[t], row_max(top[t]));
        const float fade = mx == m[t] ? 1.0f : __builtin_amdgcn_exp2f(m[t] - mx);
        m[t] = mx;
        l[t] *= fade;
#pragma unroll
        for (int c = 0; c < VC; ++c) o[t][c] *= fade;
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float base = m[t] == -__builtin_inff() ? 0.0f : m[t];  // nothing seen yet: every exponent is -infinity
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(acc[t][i >> 2][i & 3], scale2, -base));
        l[t] += p[i];
      }
      split8<false>(p, pf[t]);  // no score passes the reference by more than kSlack
    }
  }

  // o += p times channel operand c of the tile's values
  __device__ __forceinline__ void add_channel(int c, bf16x8 vf, const bf16x8 (&pf)[QT][NP]) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int p = 0; p < NP; ++p) o[t][c] = mfma(vf, pf[t][p], o[t][c]);
  }

  // One tile of keys and values.
  __device__ __forceinline__ void take(const Tile<D>& X, int32_t tb, int ok, int j) {
    f32x4 acc[QT][2];
    bf16x8 pf[QT][NP];
    score(
        [&](int u, int c) {
          // channels j D/4 + 8 c .. + 7 lie in block (8 c) / 32 of the quarter (D = 256 has two there)
          return bf16_of(X.k[u][c], scale_at(X.ks[u], D == 256 && c >= KC / 2 ? 1 : 0));
        },
        acc);
    weigh(acc, tb, ok, j, pf);
    const ValueScales V(X.vs, tb, first, end, ok, j);
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      uint32_t y[2][4];
      V.convert(X.v[0][w], X.v[1][w], y);
      add_channel(2 * w, channel(y, 0), pf);
      add_channel(2 * w + 1, channel(y, 1), pf);
    }
    if (V.any_nan) spread_nan(V.nan, tb, ok, j);
  }

  // the tokens tok + lo .. tok + hi are those that row t sees
  __device__ __forceinline__ void range(int t, int32_t tok, bool ok, int32_t& lo, int32_t& hi) const {
    hi = ok ? min(pos[t], end - 1) - tok : -1;
    lo = window > 0 ? pos[t] - window + 1 - tok : 0;
  }

  // A block of NaN reaches the rows that see its token, and no other: 0 * NaN in
  // the products would reach all of them.  So a product of what is NaN with what
  // is seen says which results it reaches.
  __device__ __forceinline__ void spread_nan(const uint32_t (&nan)[2], int32_t tb, int ok, int j) {
    const int32_t at = behind_branch(tb);  // there is no such block as a rule
    const uint32_t word[2] = {behind_branch(nan[0]), behind_branch(nan[1])};
    bf16x8 bad;
#pragma unroll
    for (int i = 0; i < 8; ++i) bad[i] = static_cast<__bf16>(word[i >> 2] >> (8 * (i & 3)) & 1u ? 1.0f : 0.0f);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      bf16x8 vis;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        int32_t lo, hi;
        range(t, at + 16 * u + 4 * j, ok >> u & 1, lo, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) vis[4 * u + i] = static_cast<__bf16>(i >= lo && i <= hi ? 1.0f : 0.0f);
      }
      const f32x4 hit = mfma(bad, vis, f32x4{0, 0, 0, 0});
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (hit[i] > 0.0f)
#pragma unroll
          for (int c = 0; c < VC; ++c) o[t][c][i] = __builtin_nanf("");
    }
  }

  // All tiles of a key range, the next tile's loads in flight during each.
  template <bool once>
  __device__ __forceinline__ void sweep(Keys<D>& K, int32_t t, int32_t t_hi, int j, uint32_t* flags) {
    Tile<D> X{}, Y{};
    int ok = t < t_hi ? K.template load<once>(t, X, flags) : 0;
    for (; t < t_hi; t += K.P.step) {
      const int next = t + K.P.step < t_hi ? K.template load<once>(t + K.P.step, Y, flags) : 0;
      const int32_t tb = K.P.begin + t * 32;
      take(X, tb, ok, j);
      X = Y;
      ok = next;
    }
  }
};

// Wavefronts a SIMD that the registers are bounded for: as many as go without
// spilling (o and q take 4 D/16 + 4 D/32 NQ registers a row tile; pieces: of the query).
constexpr int waves(int D, int pieces, int QT) { return D * QT * (1 + pieces) <= 256 ? 3 : D * QT * (1 + pieces) <= 768 ? 2 : 1; }

constexpr int kMostSplits = 128;  // parts of a key range

// query row tiles of 16 a wavefront holds where there are many rows
__host__ __device__ constexpr int row_tiles(int D, int pieces) { return D * (1 + pieces) <= 384 ? 2 : 1; }

// What a workgroup has to do: a tile of the query rows of a sequence and KV head.
// Row r is new token r / G and query head r % G of those that share the KV head.
struct Job {
  Seq q;
  int32_t s, h, tile, G, R;
};

// A job of the few-row kernel, numbered by `tiles` tiles to every sequence and head,
// or, with few_units, as the many-row kernel's units are.
__device__ __forceinline__ Job few_job(const AttendArgs& A, uint32_t job) {
  Job w;
  w.G = A.kv.q_heads / A.kv.kv_heads;
  if (A.few_units) {
    w.h = static_cast<int32_t>(job % A.kv.kv_heads);
    w.s = row_unit(A.kv, static_cast<int32_t>(job / A.kv.kv_heads), w.G, 16, &w.tile);
  } else {
    w.tile = static_cast<int32_t>(job % A.tiles);
    job /= A.tiles;
    w.h = static_cast<int32_t>(job % A.kv.kv_heads);
    w.s = static_cast<int32_t>(job / A.kv.kv_heads);
  }
  w.q = sequence(A.kv, w.s);
  w.R = w.q.count * w.G;
  if (w.R > A.few_rows) w.R = 0;  // the many-row kernel's
  if (A.few_units && (w.tile < 0 || w.tile >= (w.R + 15) >> 4)) w.R = w.tile = 0;
  return w;
}
// By one lane: every sequence has a job of tile 0 and head 0, or a unit of its number.
__device__ __forceinline__ void report(const AttendArgs& A, const Job& w, uint32_t job) {
  if (A.few_units) {
    const uint32_t s = job / A.kv.kv_heads;
    if (s < static_cast<uint32_t>(A.kv.n_seqs) && w.h == 0 && sequence(A.kv, static_cast<int32_t>(s)).bad) raise(A.kv.flags, LB_KV_BAD_LENGTH);
  } else if (w.q.bad && w.tile == 0 && w.h == 0) {
    raise(A.kv.flags, LB_KV_BAD_LENGTH);
  }
}

// Rows r0 .. r0 + 16 QT - 1 of the job into a wavefront's state; false: there are none.
template <int D, typename T, int QT>
__device__ __forceinline__ bool rows_of(const AttendArgs& A, const Job& w, int32_t r0, Rows<D, T, QT>& S, int n, int j) {
  S.scale2 = fabsf(A.scale2);
  float sign = A.scale2 < 0.0f ? -1.0f : 1.0f;
  if (A.scale2 == 0.0f) sign = 0.0f, S.scale2 = 1.0f;
  S.window = A.window;
  const bool have = r0 < w.R;
  S.p_min = have ? w.q.pos0 + r0 / w.G : -1;
  S.p_max = have ? w.q.pos0 + (min(w.R, r0 + 16 * QT) - 1) / w.G : -1;
  S.first = A.window > 0 ? max(0, S.p_min - A.window + 1) : 0;
  S.end = min(w.q.len, S.p_max + 1);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int32_t r = r0 + 16 * t + n;
    const bool live = r < w.R;
    const int32_t i = r / w.G, g = r % w.G;
    S.pos[t] = live ? w.q.pos0 + i : -1;
    S.m[t] = -__builtin_inff();
    S.l[t] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) S.o[t][c] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (live) load8(static_cast<const T*>(A.q) + (w.q.row0 + static_cast<int64_t>(i)) * A.q_stride + (w.h * w.G + g) * D + j * (D / 4) + c * 8, x);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= sign;
      split8<true>(x, S.q[t][c]);
    }
  }
  return have;
}

template <int N, typename T>
__device__ __forceinline__ void store_channels(T* dst, const float (&x)[N]) {
  if constexpr (N % 8 == 0) {
#pragma unroll
    for (int c = 0; c < N; c += 8) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[c + i];
      store8(dst + c, y);
    }
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(dst) = f32x4{x[0], x[1], x[2], x[3]};
  } else {
    typedef T T4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T4*>(dst) = T4{static_cast<T>(x[0]), static_cast<T>(x[1]), static_cast<T>(x[2]), static_cast<T>(x[3])};
  }
}

__device__ __forceinline__ float inverse(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }  // l may be NaN
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -__builtin_inff() : (m + log2f(l)) * 0.6931471805599453f; }

// The results of a wavefront's rows r0 .. r0 + 16 QT - 1 that have seen all of their keys.
template <int D, typename T, int QT>
__device__ __forceinline__ void store_rows(const AttendArgs& A, const Job& w, int32_t r0, const Rows<D, T, QT>& S, int n, int j) {
  constexpr int VC = D / 16;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float total = row_sum(S.l[t]), inv = inverse(total);
    const int32_t r = r0 + 16 * t + n;
    if (r >= w.R) continue;
    const int64_t row = w.q.row0 + static_cast<int64_t>(r / w.G);
    const int32_t hq = w.h * w.G + r % w.G;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[VC];
#pragma unroll
      for (int c = 0; c < VC; ++c) x[c] = S.o[t][c][i] * inv;
      store_channels<VC>(static_cast<T*>(A.out) + row * A.out_stride + hq * D + (4 * j + i) * (D / 16), x);
    }
    if (A.lse && j == 0) A.lse[row * A.kv.q_heads + hq] = lse_of(S.m[t], total);
  }
}

// Few query rows and short key ranges, but many of them: a wavefront takes a job on
// its own, and has nothing to join.
template <int D, typename T>
__global__ __launch_bounds__(256, waves(D, Pieces<T>::q, 1)) void k_attend_short(AttendArgs A) {
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  const uint32_t job = blockIdx.x * 4 + wave_index();
  if (job >= A.jobs) return;
  const Job w = few_job(A, job);
  if (lane == 0) report(A, w, job);
  Rows<D, T, 1> S;
  if (!rows_of<D, T, 1>(A, w, w.tile * 16, S, n, j)) return;
  Keys<D> K(A.kv, w.s, w.h, S.first, S.end, 1, n, j);
  S.template sweep<false>(K, 0, S.end > K.P.begin ? (S.end - K.P.begin + 31) >> 5 : 0, j, A.kv.flags);
  store_rows<D, T, 1>(A, w, w.tile * 16, S, n, j);
}

// Few query rows: a workgroup takes 16 rows and one part of their key range; its
// four wavefronts take every fourth tile and join at the end.  once: nobody else
// reads the keys, which then leave the caches to others (4 x 110 000 keys of 8 heads:
// 92 us, else 100).
template <int D, typename T, bool once>
__global__ __launch_bounds__(256, waves(D, Pieces<T>::q, 1)) void k_attend(AttendArgs A) {
  constexpr int VC = D / 16;
  const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, j = lane >> 4;
  const uint32_t job = blockIdx.x / A.splits;
  const int32_t split = static_cast<int32_t>(blockIdx.x % A.splits);
  const Job w = few_job(A, job);
  if (split == 0 && threadIdx.x == 0) report(A, w, job);
  Rows<D, T, 1> S;
  if (!rows_of<D, T, 1>(A, w, w.tile * 16, S, n, j)) return;
  Keys<D> K(A.kv, w.s, w.h, S.first, S.end, 4, n, j);
  const int32_t tiles = S.end > K.P.begin ? (S.end - K.P.begin + 31) >> 5 : 0;
  const int32_t per = (tiles + A.splits - 1) / A.splits;
  S.template sweep<once>(K, split * per + wave, min(tiles, (split + 1) * per), j, A.kv.flags);
  const float l = row_sum(S.l[0]);

  // join the four wavefronts
  __shared__ float part[4][VC * 4][64];
  __shared__ float pm[4][16], pl[4][16];
#pragma unroll
  for (int c = 0; c < VC; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][4 * c + i][lane] = S.o[0][c][i];
  if (j == 0) pm[wave][n] = S.m[0], pl[wave][n] = l;
  __syncthreads();
  const float M = fmaxf(fmaxf(pm[0][n], pm[1][n]), fmaxf(pm[2][n], pm[3][n]));
  const float base = M == -__builtin_inff() ? 0.0f : M;
  float wgt[4], L = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    wgt[k] = __builtin_amdgcn_exp2f(pm[k][n] - base);
    L += wgt[k] * pl[k][n];
  }
  const int32_t r = w.tile * 16 + n;
  if (r >= w.R) return;
  const int64_t row = w.q.row0 + static_cast<int64_t>(r / w.G);
  const int32_t hq = w.h * w.G + r % w.G;
  // wavefront i writes the rows 4 j + i of the results: D/16 adjacent channels a lane
  const int i = wave;
  float x[VC];
#pragma unroll
  for (int c = 0; c < VC; ++c) {
    x[c] = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[c] += wgt[k] * part[k][4 * c + i][lane];
  }
  const int32_t ch = (4 * j + i) * (D / 16);
  if (A.splits > 1) {
    const int64_t at = (static_cast<int64_t>(job) * A.part_rows + n) * A.splits + split;
    store_channels<VC>(A.part + at * D + ch, x);
    if (i == 0 && j == 0) {
      float* sums = A.part + A.part_sums + at * 2;
      sums[0] = M, sums[1] = L;
    }
    return;
  }
  const float inv = inverse(L);
#pragma unroll
  for (int c = 0; c < VC; ++c) x[c] *= inv;
  store_channels<VC>(static_cast<T*>(A.out) + row * A.out_stride + hq * D + ch, x);
  if (A.lse && i == 0 && j == 0) A.lse[row * A.kv.q_heads + hq] = lse_of(base, L);
}

// Many query rows: each of the four wavefronts has 16 QT rows of its own, and all
// take the same tiles.  A tile is converted to bf16 operands once, a quarter by
// each wavefront, and goes through LDS in the order in which lanes read it.  While
// the probabilities of tile t are computed, its values come from LDS; the products
// with them hide the reading of the keys of t + 1, whose scores follow.  Later keys
// and values are converted meanwhile, and what the step after needs is on its way
// from memory.  A ring of 2 A tiles has a barrier every A tiles: at step t the keys
// of t + 1 and the values of t are read, made A steps or more before, and those of t
// + 1 + A and t + A are made, in places that were last read A steps or more before.
// Six prompts of 65..2048 tokens over 130..4096, 32 heads of 128 on 8, bf16: 408 us,
// 570 TFLOP/s; vector instructions are issued in 54 % of the SIMD cycles (a lane's
// eight scores of a row take 8 products, exponentials and sums each, and 24 for their
// two pieces), matrix ones run in 36 %, and two wavefronts a SIMD do not cover each
// other's waits.
template <int D>
struct Shared {
  static constexpr int KC = D / 32, VC = D / 16;
  static constexpr int A = D <= 128 ? 2 : 1, N = 2 * A;
  bf16x8 key[N][2 * KC][64], value[N][VC][64];  // [tile % N][half and channels, or channel][lane]
  uint32_t nan[N][2][64];
  int32_t any_nan[N];
};
static_assert(sizeof(Shared<64>) <= 80 << 10 && sizeof(Shared<128>) <= 80 << 10 && sizeof(Shared<256>) <= 80 << 10, "two workgroups a CU");

template <int D>
struct Maker {
  static constexpr int F = D / 64, W = F > 1 ? F / 2 : 1;  // operands of keys and of values a wavefront makes; words of values
  Pages P;
  const uint8_t* base;
  int64_t page_bytes;
  uint32_t k_at, v_at, ks_at, vs_at;
  int u;  // the half whose keys are this wavefront's
  uint32_t k[F], v[2][W], ks, vs[2];
  int ok;                    // the halves there are of the tile whose values are held
  const uint8_t* half[2];    // where the halves start of the tile whose keys are held: codes and, P D bytes on, scales
  const uint8_t* scales[2];
  int there = 0;             // the halves there are of that tile

  __device__ __forceinline__ Maker(const KvArgs& A, int32_t s, int32_t h, int32_t first, int32_t end, int wave, int n, int j)
      : P(A, s, first, end, 1), u(wave >> 1), ks(0), ok(0) {
    const int32_t T = 1 << A.page_shift, block = T * (D + D / 16), c0 = (wave & 1) * F, w0 = D == 64 ? wave >> 1 : wave * W;
    base = A.pages + static_cast<int64_t>(h) * block;
    page_bytes = static_cast<int64_t>(block) * A.kv_heads;
    k_at = n * (D / 2) + j * (D / 8) + c0 * 4;
    v_at = T * (D / 2) + j * (D * 2) + n * (D / 8) + w0 * 4;
    ks_at = T * D + n * (D / 32) + (j * (D / 4) + c0 * 8) / 32;
    vs_at = T * D + T * (D / 32) + (j * (D / 32) + n * D / 512) * 4;
#pragma unroll
    for (int i = 0; i < F; ++i) k[i] = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) v[0][i] = v[1][i] = 0;
    vs[0] = vs[1] = 0;
  }

  __device__ __forceinline__ void load_keys(int32_t t, uint32_t* flags) {
    int32_t page[2];
    P.of(t, page, flags);
    there = (page[0] >= 0 ? 1 : 0) | (page[1] >= 0 ? 2 : 0);
    const int32_t slot = P.slot(t, 0), next = P.slot(t, 1);
    half[0] = base + page[0] * page_bytes;
    half[1] = page[1] == page[0] ? half[0] : base + page[1] * page_bytes;
    scales[0] = half[0] + slot * (D / 32), scales[1] = half[1] + next * (D / 32);
    half[0] += slot * (D / 2), half[1] += next * (D / 2);
    if (there >> u & 1) {  // else what the registers hold stays unseen
      load_words<F>((u ? half[1] : half[0]) + k_at, k);
      ks = (u ? scales[1] : scales[0])[ks_at];
    }
  }
  // of the tile that load_keys loaded last
  __device__ __forceinline__ void load_values() {
    ok = there;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (!(ok >> x & 1)) continue;
      load_words<W>(half[x] + v_at, v[x]);
      vs[x] = *reinterpret_cast<const uint32_t*>(scales[x] + vs_at);
    }
  }

  // what has been loaded, into buffer b; tb: the tile's first token
  __device__ __forceinline__ void make_keys(Shared<D>& L, int b, int wave, int lane) const {
    const float s = scale_of(ks);
#pragma unroll
    for (int i = 0; i < F; ++i) L.key[b][wave * F + i][lane] = bf16_of(k[i], s);
  }
  __device__ __forceinline__ void make_values(Shared<D>& L, int b, int32_t tb, int wave, int lane) const {
    const ValueScales V(vs, tb, P.first, P.end, ok, lane >> 4);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      uint32_t y[2][4];
      V.convert(v[0][i], v[1][i], y);
      if constexpr (D == 64) {
        L.value[b][wave][lane] = channel(y, wave & 1);
      } else {
        L.value[b][wave * F + 2 * i][lane] = channel(y, 0);
        L.value[b][wave * F + 2 * i + 1][lane] = channel(y, 1);
      }
    }
    if (wave == 0) {  // its lanes have the scales of all blocks
      if (V.any_nan) L.nan[b][0][lane] = V.nan[0], L.nan[b][1][lane] = V.nan[1];
      if (lane == 0) L.any_nan[b] = V.any_nan;
    }
  }
};

// Operands that the many-row kernel reads ahead: as many of N as the registers hold beside its state.
template <int D, typename T, int QT>
constexpr int ahead(int N) {
  const int state = 4 * QT * (D / 16 + D / 32 * Pieces<T>::q + 2 + Pieces<T>::p) + 56, room = (256 - state) / 8;
  return room >= N ? N : room >= N / 2 ? N / 2 : room >= 4 ? 4 : 2;
}

template <int D, typename T, int QT>
__global__ __launch_bounds__(256, waves(D, Pieces<T>::q, QT)) void k_attend_rows(AttendArgs A) {
  constexpr int KC = D / 32, VC = D / 16, NP = Pieces<T>::p, per = 64 * QT;
  constexpr int KA = ahead<D, T, QT>(2 * KC), VA = ahead<D, T, QT>(VC);
  __shared__ Shared<D> L;
  const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, j = lane >> 4;
  if (A.few_rows == 0) check_sequence(A.kv, blockIdx.x);
  Job w;
  w.G = A.kv.q_heads / A.kv.kv_heads;
  w.h = static_cast<int32_t>(blockIdx.x % A.kv.kv_heads);
  w.s = row_unit(A.kv, static_cast<int32_t>(blockIdx.x / A.kv.kv_heads), w.G, per, &w.tile);
  w.q = sequence(A.kv, w.s);
  w.R = w.q.count * w.G;
  if (w.R <= A.few_rows) return;  // the few-row kernel's
  const int32_t tiles_of_rows = (w.R + per - 1) / per;
  if (w.tile < 0 || w.tile >= tiles_of_rows) return;
  w.tile = tiles_of_rows - 1 - w.tile;  // the last rows see most keys: they go first
  // a wavefront without rows goes along, and sees nothing
  Rows<D, T, QT> S;
  const bool have = rows_of<D, T, QT>(A, w, (w.tile * 4 + wave) * 16 * QT, S, n, j);
  // the key range of all four wavefronts' rows
  const int32_t p_min = w.q.pos0 + w.tile * per / w.G, p_max = w.q.pos0 + (min(w.R, (w.tile + 1) * per) - 1) / w.G;
  const int32_t first = A.window > 0 ? max(0, p_min - A.window + 1) : 0, begin = first & ~31, end = min(w.q.len, p_max + 1);
  const int32_t tiles = end > begin ? (end - begin + 31) >> 5 : 0;
  if (tiles > 0) {
    Maker<D> M(A.kv, w.s, w.h, first, end, wave, n, j);
    f32x4 acc[QT][2];
    bf16x8 kf[KA], vf[VA];
    const auto read_keys = [&](int b) {
#pragma unroll
      for (int i = 0; i < KA; ++i) kf[i] = L.key[b][i][lane];
    };
    const auto score = [&](int b) {
      S.score([&](int u, int c) { return u * KC + c < KA ? kf[u * KC + c] : L.key[b][u * KC + c][lane]; }, acc);
    };
    constexpr int S_A = Shared<D>::A, N = Shared<D>::N;
    int ok[S_A + 1];  // the halves there are of tiles t .. t + A
#pragma unroll
    for (int i = 0; i <= S_A; ++i) {
      M.load_keys(min(i, tiles - 1), A.kv.flags);
      M.make_keys(L, i, wave, lane);
      M.load_values();
      ok[i] = M.ok;
      if (i < S_A) M.make_values(L, i, begin + 32 * i, wave, lane);
    }
    M.load_keys(min(S_A + 1, tiles - 1), A.kv.flags);
    __syncthreads();
    read_keys(0);
    score(0);
    __syncthreads();  // before other keys go where those of tile 0 are
    // past the last tile the last one is made again, and nobody reads it
#pragma unroll S_A
    for (int32_t t = 0; t < tiles; ++t) {
      const int b = t & (N - 1);
      const int32_t tb = begin + t * 32;
#pragma unroll
      for (int c = 0; c < VA; ++c) vf[c] = L.value[b][c][lane];
      const int32_t flag = L.any_nan[b];
      M.make_keys(L, (t + 1 + S_A) & (N - 1), wave, lane);
      M.make_values(L, (t + S_A) & (N - 1), tb + 32 * S_A, wave, lane);
      M.load_values();
      M.load_keys(min(t + 2 + S_A, tiles - 1), A.kv.flags);
      bf16x8 pf[QT][NP];
      const int here = ok[0];
      S.weigh(acc, tb, here, j, pf);
#pragma unroll
      for (int i = 0; i < S_A; ++i) ok[i] = ok[i + 1];
      ok[S_A] = M.ok;
      const bool any_nan = __builtin_amdgcn_readfirstlane(flag) != 0;
      __builtin_amdgcn_sched_barrier(0);
      read_keys((t + 1) & (N - 1));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < VC; ++c) S.add_channel(c, c < VA ? vf[c] : L.value[b][c][lane], pf);
      if (any_nan) {
        const uint32_t nan[2] = {L.nan[b][0][lane], L.nan[b][1][lane]};
        S.spread_nan(nan, tb, here, j);
      }
      score((t + 1) & (N - 1));
      if (S_A == 1 || (t & (S_A - 1)) == S_A - 1) __syncthreads();
    }
  }
  if (have) store_rows<D, T, QT>(A, w, (w.tile * 4 + wave) * 16 * QT, S, n, j);
}

// Joins the parts of a row's key range: a workgroup per row of the few-row
// kernel's jobs.  A group of D/4 lanes takes a part, 16 B a lane, all parts' loads
// on their way at a time.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs A) {
  constexpr int L = D / 4, groups = 256 / L;
  const uint32_t job = blockIdx.x / A.part_rows;
  const Job w = few_job(A, job);
  const int32_t r = w.tile * 16 + static_cast<int32_t>(blockIdx.x % A.part_rows);
  if (r >= w.R) return;
  const int lane = threadIdx.x & 63, g = threadIdx.x / L, c = threadIdx.x % L;
  const int64_t row = w.q.row0 + static_cast<int64_t>(r / w.G);
  const int32_t hq = w.h * w.G + r % w.G;
  const float* parts = A.part + static_cast<int64_t>(blockIdx.x) * A.splits * D;
  const float* sums = A.part + A.part_sums + static_cast<int64_t>(blockIdx.x) * A.splits * 2;
  f32x4 p[kMostSplits / groups];
#pragma unroll
  for (int k = 0; k < kMostSplits / groups; ++k)
    p[k] = g + k * groups < A.splits ? *reinterpret_cast<const f32x4*>(parts + (g + k * groups) * D + 4 * c) : f32x4{0, 0, 0, 0};
  // lane i: the sums of parts i and 64 + i
  float m[2], l[2], M = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const bool have = lane + 64 * k < A.splits;
    m[k] = have ? sums[2 * (lane + 64 * k)] : -__builtin_inff();
    l[k] = have ? sums[2 * (lane + 64 * k) + 1] : 0.0f;
    M = fmaxf(M, m[k]);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) M = fmaxf(M, __shfl_xor(M, d));
  const float base = M == -__builtin_inff() ? 0.0f : M;
  float total = 0.0f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    m[k] = __builtin_amdgcn_exp2f(m[k] - base);
    total += m[k] * l[k];
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
  f32x4 x{0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < kMostSplits / groups; ++k) {
    const int at = g + k * groups;
    const float f = __shfl(at < 64 ? m[0] : m[1], at & 63);  // parts that do not exist have 0
    x += f * p[k];
  }
  __shared__ f32x4 joined[256];
  joined[threadIdx.x] = x;
  __syncthreads();
  const float inv = inverse(total);
  if (threadIdx.x < L) {
#pragma unroll
    for (int k = 1; k < groups; ++k) x += joined[k * L + threadIdx.x];
    const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
    store_channels<4>(static_cast<T*>(A.out) + row * A.out_stride + hq * D + 4 * threadIdx.x, y);
  }
  if (A.lse && threadIdx.x == 0) A.lse[row * A.kv.q_heads + hq] = lse_of(base, total);
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
  if (A.units) {
    const int64_t blocks = A.units * A.kv.kv_heads;
    k_attend_rows<D, T, row_tiles(D, Pieces<T>::q)><<<dim3(static_cast<unsigned>(blocks)), 256, 0, st>>>(A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || A.few_rows == 0) return e;
  }
  const int64_t jobs = A.jobs;
  if (A.alone) {
    k_attend_short<D, T><<<dim3(static_cast<unsigned>((jobs + 3) / 4)), 256, 0, st>>>(A);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>(jobs * A.splits));
  if (A.tiles == 1 && A.splits > 1)
    k_attend<D, T, true><<<grid, 256, 0, st>>>(A);
  else
    k_attend<D, T, false><<<grid, 256, 0, st>>>(A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.splits == 1) return e;
  k_attend_join<D, T><<<dim3(static_cast<unsigned>(jobs * A.part_rows)), 256, 0, st>>>(A);
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

constexpr int64_t kLeastGroups = 600;  // of 128 rows

// How a call is cut up.  Sequences with at most few_rows query rows a KV head: tiles
// of 16 rows, as many for each as max_new may need or, where those are more, numbered
// by the rows there are (1024 single tokens beside a prompt of 500, 32 heads of 128 on
// 8, bf16: 110 us, else 1462; two sequences of up to 100 new tokens: 8.0, else 7.6), and
// parts of the key range so that about three workgroups a CU exist (as many as are
// resident with 128 channels in bf16: 4 x 110 000 keys of 8 heads take 92 us with them,
// 110 with two or eight, 100 with six), each with 16 tiles of keys at least; where there
// are many such jobs with at most 16 tiles of keys, a wavefront takes one alone (1024
// sequences of 3 to 256 keys, 4 heads of 64: 19 us, else 26).  The others: a workgroup
// takes the rows of its four wavefronts, and the workgroups are numbered as append's
// units are, so that a ragged batch has no more than one idle one a sequence and head.
// A batch that may hold both gets both kernels, each of which leaves the other's
// sequences alone.  The many-row kernel does an eighth of the conversions, but it has no
// parts of keys: with fewer rows than fill the chip (512 workgroups of 128 rows are
// resident) all goes to the other (8 KV heads of 128 channels, 4 query heads each, bf16:
// 100 new tokens of 20 000, 25 groups of 128 rows, 110 us, else 907; 1000 of 5000, 250
// groups, 175 us, else 237; 3000 of 3000, 750 groups, 191 us, else 148).
AttendPlan attend_plan(const KvArgs& kv, int head_dim, int dtype) {
  AttendPlan p{};
  const int64_t G = kv.q_heads / kv.kv_heads, rows = kv.max_new * G;
  const int pieces = dtype == LB_BF16 ? Pieces<__bf16>::q : dtype == LB_F16 ? Pieces<_Float16>::q : Pieces<float>::q;
  const int64_t units = kv.n_rows * G / (4 * 16 * row_tiles(head_dim, pieces)) + kv.n_seqs;
  const int64_t most_units = kv.n_rows * G / (4 * 16 * row_tiles(head_dim, Pieces<float>::q)) + kv.n_seqs;
  p.splits = 1;
  p.few_rows = 0x7FFFFFFF;
  if (rows > 64 && kv.n_rows * G * kv.kv_heads >= 128 * kLeastGroups) {
    p.units = units;
    p.groups = most_units * kv.kv_heads;
    p.few_rows = kv.n_seqs == 1 ? 0 : 64;
    if (p.few_rows == 0) return p;
  }
  const int64_t most = rows < p.few_rows ? rows : p.few_rows;
  p.tiles = static_cast<int32_t>((most + 15) / 16);
  p.part_rows = static_cast<int32_t>(most < 16 ? most : 16);
  const int64_t few_units = kv.n_rows * G / 16 + kv.n_seqs;
  const bool numbered = few_units < static_cast<int64_t>(kv.n_seqs) * p.tiles;
  p.few_units = numbered ? few_units : 0;
  const int64_t jobs = p.jobs = (numbered ? few_units : static_cast<int64_t>(kv.n_seqs) * p.tiles) * kv.kv_heads;
  const int64_t tokens = static_cast<int64_t>(kv.max_pages) << kv.page_shift;
  p.alone = tokens <= 512 && jobs > 2048;
  int64_t s = (768 + jobs - 1) / jobs;
  s = s < tokens / 512 ? s : tokens / 512;
  p.splits = static_cast<int32_t>(s < 1 ? 1 : s > kMostSplits ? kMostSplits : s);
  p.groups = p.groups > jobs * p.splits ? p.groups : jobs * p.splits;
  if (p.splits > 1) {
    p.part_sums = jobs * p.part_rows * p.splits * head_dim;
    p.part_floats = p.part_sums + jobs * p.part_rows * p.splits * 2;
  }
  return p;
}

}  // namespace lb
