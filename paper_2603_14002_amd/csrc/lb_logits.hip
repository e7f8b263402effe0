// Penalties, biases and masks on logits, and their log-probabilities.
//
// A row is read once for its maximum and sum (kept together, the sum rescaled
// when the maximum grows) and once more where its log-probabilities are wanted.
//
// Long rows: a workgroup takes a part of a row, 16 B a lane at a time.  The
// classes that a history or a bias list names are few: they are left out of that
// sweep, as the masked ones are, by one bit a class in LDS, and handled on their
// own from a hash table of at most LB_MAX_RULE_IDS entries, so the sweep has no
// branch for them.  4096 rows of 125 002 in bf16, scores alone: 192 us, 5.3 TB/s,
// bound by memory (205 us where what is read once stays in the caches).
//
// Short rows (up to 512 classes): 16 or 64 lanes hold a row in registers and
// read it once, the next one on its way.  128 000 rows of 41 in fp32: 14.2 us, 3.0
// TB/s, bound by the two reductions of a row, each four dependent steps.
#include <hip/hip_runtime.h>

#include "lb_scorer.h"

namespace lb {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__bf16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float as_float(_Float16 x) { return static_cast<float>(x); }

// the mask of a row where there are masks; none if outside 0 .. mask_rows - 1
__device__ __forceinline__ int64_t mask_index(const LogitArgs& A, int64_t row) {
  return A.r.mask_row ? A.r.mask_row[row] : A.r.mask_rows == 1 ? 0 : row;
}
__device__ __forceinline__ const uint32_t* mask_of(const LogitArgs& A, int64_t row) {
  if (!A.r.mask) return nullptr;
  const int64_t k = mask_index(A, row);
  return k >= 0 && k < A.r.mask_rows ? A.r.mask + k * ((A.classes + 31) / 32) : nullptr;
}

// The rules for one class up to the temperature, in the order that the header
// gives.  The division by the repetition penalty is a product with its rounded
// reciprocal: one rounding of 2^-24 more.
struct Rules {
  float repetition, inv_repetition, presence, frequency;
  __device__ __forceinline__ explicit Rules(const lb_logit_rules& r)
      : repetition(r.repetition), inv_repetition(1.0f / r.repetition), presence(r.presence), frequency(r.frequency) {}
  __device__ __forceinline__ float operator()(float x, int32_t count, float bias) const {
    if (count) x = x * (x > 0.0f ? inv_repetition : repetition) - presence - frequency * static_cast<float>(count);
    return x + bias;
  }
};

// The temperature goes into the exponent: with k = log2(e) / temperature, rounded, a
// term is 2^(k (x - m)), m the largest logit before the temperature.  What k lacks
// (2^-24 of it, as the rounded quotient by the temperature would) is that part of a
// difference between logits, not of the logits; and no logit is scaled, so those of
// the type's lowest value stay finite.  A row's sum is (m, l); nothing yet: (-inf, 0).
struct Sum {
  float m, l;
};
// what exponents are taken relative to: an infinite maximum would make inf - inf of them
__device__ __forceinline__ float safe(float m) { return __builtin_isinf(m) ? 0.0f : m; }
__device__ __forceinline__ float term(float x, float base, float k) { return __builtin_amdgcn_exp2f((x - base) * k); }
__device__ __forceinline__ void join(Sum& a, float m2, float l2, float k) {
  const float m = fmaxf(a.m, m2), base = safe(m);
  a.l = a.l * term(a.m, base, k) + l2 * term(m2, base, k);
  a.m = m;
}
// n logits at once: one rescaling of the sum
template <int n>
__device__ __forceinline__ void add(Sum& a, const float (&x)[n], float k) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < n; ++i) m = fmaxf(m, x[i]);
  const float base = safe(m);
  float l = a.l * term(a.m, base, k);
#pragma unroll
  for (int i = 0; i < n; ++i) l += term(x[i], base, k);
  a.l = l;
  a.m = m;
}
// sum or maximum over the 16 or 64 lanes of a row, by moves within a row of 16
// lanes (pairs, quads, and mirrored halves, where each half has one value already)
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Plus {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
template <int ctrl>
__device__ __forceinline__ float moved(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), ctrl, 0xF, 0xF, true));
}
template <int L, typename F>
__device__ __forceinline__ float over_lanes(float x, F f) {
  x = f(x, moved<0xB1>(x));   // lanes 1 0 3 2
  x = f(x, moved<0x4E>(x));   // lanes 2 3 0 1
  x = f(x, moved<0x141>(x));  // row_half_mirror
  x = f(x, moved<0x140>(x));  // row_mirror
  if constexpr (L == 64) {
    x = f(x, __shfl_xor(x, 16));
    x = f(x, __shfl_xor(x, 32));
  }
  return x;
}
__device__ __forceinline__ Sum block_sum(Sum s, float k) {
  __shared__ float sm[4], sl[4];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float m2 = __shfl_xor(s.m, d), l2 = __shfl_xor(s.l, d);
    join(s, m2, l2, k);
  }
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s.m, sl[threadIdx.x >> 6] = s.l;
  __syncthreads();
  Sum t{sm[0], sl[0]};
#pragma unroll
  for (int w = 1; w < 4; ++w) join(t, sm[w], sl[w], k);
  return t;
}
// The log-sum-exp as its reference m (a logit before the temperature) and the rest:
// log p = (x - m) / temperature - rest stays right where m is so large that m + rest
// is m.  The quotient is a product with the rounded reciprocal.
struct Lse {
  float m, rest, inv;
  __device__ __forceinline__ float value() const { return fmaf(m, inv, rest); }
};
__device__ __forceinline__ Lse log_sum(Sum s, float temperature) {
  return {safe(s.m), s.l == 0.0f ? -__builtin_inff() : log2f(s.l) * kLn2, 1.0f / temperature};
}
__device__ __forceinline__ float log_prob(float x, Lse lse) { return x == -__builtin_inff() ? x : fmaf(x - lse.m, lse.inv, -lse.rest); }

// xt: the target's logit after the rules up to the temperature
__device__ __forceinline__ void finish(const LogitArgs& A, int64_t row, Lse lse, float xt) {
  if (A.lse) A.lse[row] = lse.value();
  if (!A.score) return;
  const int32_t t = A.target[row];
  A.score[row] = t < 0 ? 0.0f : t >= A.classes ? __builtin_nanf("") : log_prob(xt, lse);
}

// ------------------------------------------------------------------ long rows

constexpr int kPartClasses = 131072;  // classes of one part at most: 16 KB of bits, eight workgroups a CU

struct Slot {
  int32_t id;     // -1: empty
  int32_t count;  // occurrences in the history
  int32_t entry;  // the entry that answers for the class: its last bias (kBias + place), else its first occurrence (history_width - place)
  float x;        // the class's logit after the rules up to the temperature
};
constexpr int32_t kBias = LB_MAX_RULE_IDS + 1;

// A part of a row: the classes lo .. hi - 1, in chunks of eight that start at
// 16-B aligned logits (the first and last may be cut short).  bit 8 c + i of
// `open` is set where class i of chunk c is in the part, allowed by the mask and
// not named.
template <typename T>
struct Part {
  const T* src;     // logits of the row
  int32_t lo, hi, first;  // class at bit 0
  int32_t chunks;
  uint8_t* open;
  Slot* table;
  int32_t slots;
  bool sparse;  // some bit may be clear (other than outside the part)
  float k;
  const int32_t *past, *biased;  // the row's lists
  int32_t H, W;

  __device__ __forceinline__ void start(const LogitArgs& A, int64_t row, int32_t part, int32_t parts, int32_t n_slots, uint32_t* shared) {
    const int32_t per = (A.classes + parts - 1) / parts;
    lo = min(A.classes, part * per);
    hi = min(A.classes, lo + per);
    src = static_cast<const T*>(A.logits) + row * A.stride;
    first = lo - static_cast<int32_t>((reinterpret_cast<uintptr_t>(src + lo) & 15) / sizeof(T));
    chunks = (hi - first + 7) >> 3;
    const Rules rules(A.r);
    k = kLog2e / A.r.temperature;
    slots = n_slots;
    const uint32_t* mask = mask_of(A, row);
    sparse = mask || slots;
    open = reinterpret_cast<uint8_t*>(shared);
    const int32_t words = (chunks + 3) >> 2;
    table = reinterpret_cast<Slot*>(shared + ((words + 3) & ~3));
    if (!sparse) return;
    for (int32_t i = threadIdx.x; i < words; i += 256) {
      uint32_t w = 0xFFFFFFFFu;
      if (mask) {
        // classes first + 32 i .. + 31 of the mask (first may lie before class 0: those bits are not looked at)
        const int32_t c = first + 32 * i, at = c >> 5, sh = c & 31, last = (A.classes - 1) >> 5;
        const uint32_t a = at >= 0 ? mask[min(at, last)] : 0, b = at + 1 <= last ? mask[at + 1] : 0;
        w = sh ? a >> sh | b << (32 - sh) : a;
      }
      shared[i] = w;
    }
    if (!slots) {
      __syncthreads();
      return;
    }
    for (int32_t i = threadIdx.x; i < slots; i += 256) table[i] = Slot{-1, 0, 0, 0.0f};
    __syncthreads();
    H = A.r.history_width, W = A.r.bias_width;
    const int64_t list = A.r.bias_per_row ? row * W : 0;
    past = A.r.history + row * H, biased = A.r.bias_ids + list;
    for (int32_t i = threadIdx.x; i < H; i += 256) put(past[i], 1, H - i);
    for (int32_t i = threadIdx.x; i < W; i += 256) put(biased[i], 0, kBias + i);
    __syncthreads();
    for (int32_t i = threadIdx.x; i < slots; i += 256) {
      Slot& s = table[i];
      if (s.id < 0) continue;
      const int32_t at = s.id - first;
      if (shared[at >> 5] >> (at & 31) & 1u) {
        atomicAnd(&shared[at >> 5], ~(1u << (at & 31)));
        s.x = rules(as_float(src[s.id]), s.count, s.entry >= kBias ? A.r.bias_values[list + s.entry - kBias] : 0.0f);
      } else {
        s.x = -__builtin_inff();  // masked
      }
    }
    __syncthreads();
  }

  __device__ __forceinline__ bool inside(int32_t id) const { return id >= lo && id < hi; }
  __device__ __forceinline__ uint32_t first_slot(int32_t id) const { return (static_cast<uint32_t>(id) * 2654435761u) >> (__builtin_clz(slots) + 1); }
  __device__ __forceinline__ void put(int32_t id, int32_t count, int32_t entry) {
    if (!inside(id)) return;
    uint32_t at = first_slot(id);
    for (;;) {
      const int32_t was = atomicCAS(&table[at].id, -1, id);
      if (was == -1 || was == id) break;
      at = (at + 1) & (slots - 1);
    }
    if (count) atomicAdd(&table[at].count, count);
    atomicMax(&table[at].entry, entry);
  }
  // the slot of a class, or the empty one where it would be (half of the slots are empty at least)
  __device__ __forceinline__ uint32_t find(int32_t id) const {
    uint32_t at = first_slot(id);
    while (table[at].id != id && table[at].id >= 0) at = (at + 1) & (slots - 1);
    return at;
  }

  // the logits of chunk c, -infinity where its bits are clear; false: the chunk is cut short
  __device__ __forceinline__ bool load(int32_t c, float (&x)[8]) const {
    const int32_t w = first + 8 * c;
    const bool whole = w >= lo && w + 8 <= hi;
    if (whole) {
      load8(src + w, x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = w + i >= lo && w + i < hi ? as_float(src[w + i]) : -__builtin_inff();
    }
    if (sparse) mask(x, open[c]);
    return whole;
  }
  static __device__ __forceinline__ void mask(float (&x)[8], uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t keep = static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - i)) >> 31);  // all ones where the bit is set
      x[i] = __uint_as_float((__float_as_uint(x[i]) & keep) | (0xFF800000u & ~keep));
    }
  }

  // once: the row is not read again
  template <bool once>
  __device__ __forceinline__ Sum sum(int32_t target, float* xt) const {
    Sum s{-__builtin_inff(), 0.0f};
    // whole chunks, two at a time: two loads on their way, and one rescaling for both
    int32_t c = threadIdx.x;
    const int32_t last = (hi - first) >> 3;  // chunks that end inside
    if (c == 0 && first < lo && c < chunks) one(s, c), c += 256;
    for (; c + 256 < last; c += 512) {
      float x[16];
      if constexpr (once) {
        load8_nt(src + first + 8 * c, *reinterpret_cast<float(*)[8]>(x));
        load8_nt(src + first + 8 * (c + 256), *reinterpret_cast<float(*)[8]>(x + 8));
      } else {
        load8(src + first + 8 * c, *reinterpret_cast<float(*)[8]>(x));
        load8(src + first + 8 * (c + 256), *reinterpret_cast<float(*)[8]>(x + 8));
      }
      if (sparse) {
        mask(*reinterpret_cast<float(*)[8]>(x), open[c]);
        mask(*reinterpret_cast<float(*)[8]>(x + 8), open[c + 256]);
      }
      add(s, x, k);
    }
    for (; c < chunks; c += 256) one(s, c);
    // the named classes, each by the thread of the entry that answers for it: the order of the sum is the lists',
    // not that in which the wavefronts came to the table
    if (slots) {
      for (int32_t i = threadIdx.x; i < H; i += 256) named(s, past[i], H - i);
      for (int32_t i = threadIdx.x; i < W; i += 256) named(s, biased[i], kBias + i);
    }
    if (threadIdx.x == 0 && inside(target)) {
      const int32_t at = target - first;
      if (!sparse || open[at >> 3] >> (at & 7) & 1)
        *xt = as_float(src[target]);
      else if (slots && table[find(target)].id == target)
        *xt = table[find(target)].x;
    }
    return s;
  }
  __device__ __forceinline__ void named(Sum& s, int32_t id, int32_t entry) const {
    if (!inside(id)) return;
    const Slot& at = table[find(id)];
    if (at.entry != entry) return;
    const float x[1] = {at.x};
    add(s, x, k);
  }
  __device__ __forceinline__ void one(Sum& s, int32_t c) const {
    float x[8];
    load(c, x);
    add(s, x, k);
  }

  __device__ __forceinline__ void write(float* dst, Lse lse) const {
    const bool even = ((reinterpret_cast<uintptr_t>(dst + first) & 15) == 0);
    for (int32_t c = threadIdx.x; c < chunks; c += 256) {
      float x[8];
      const bool whole = load(c, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = log_prob(x[i], lse);
      const int32_t w = first + 8 * c;
      if (whole && even) {
        store8(dst + w, x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (w + i >= lo && w + i < hi) dst[w + i] = x[i];
      }
    }
    if (!slots) return;
    __syncthreads();  // the named classes' places have been written above, as masked
    for (int32_t i = threadIdx.x; i < slots; i += 256)
      if (table[i].id >= 0) dst[table[i].id] = log_prob(table[i].x, lse);
  }
};

// One part of a row: its sum, and all the rest where the row has one part.  The
// parts' sums are kept at part[row][split] = (m, l), the target's logit after them.
template <typename T, bool once>
__global__ __launch_bounds__(256) void k_logits(LogitArgs A, int32_t slots) {
  extern __shared__ uint32_t shared[];
  __shared__ float xt;
  const int64_t row = A.row0 + blockIdx.x / A.splits;
  const int32_t part = static_cast<int32_t>(blockIdx.x % A.splits);
  Part<T> P;
  if (threadIdx.x == 0) xt = -__builtin_inff();
  P.start(A, row, part, A.splits, slots, shared);
  const int32_t target = A.score ? A.target[row] : -1;
  if (!P.sparse) __syncthreads();  // xt
  Sum s = block_sum(P.template sum<once>(target, &xt), P.k);  // its barrier also shows xt to all
  if (A.splits > 1) {
    if (threadIdx.x == 0) {
      A.part[2 * (row * A.splits + part)] = s.m;
      A.part[2 * (row * A.splits + part) + 1] = s.l;
      if (target >= P.lo && target < P.hi) A.part[2 * A.rows * A.splits + row] = xt;
    }
    return;
  }
  const Lse lse = log_sum(s, A.r.temperature);
  if (threadIdx.x == 0) finish(A, row, lse, xt);
  if (A.logprobs) P.write(A.logprobs + row * A.out_stride, lse);
}

// Rows of several parts: joins the sums, then writes the part's log-probabilities.
template <typename T>
__global__ __launch_bounds__(256) void k_logits_join(LogitArgs A, int32_t slots) {
  extern __shared__ uint32_t shared[];
  const int32_t parts = A.logprobs ? A.splits : 1;
  const int64_t row = A.row0 + blockIdx.x / parts;
  const int32_t part = static_cast<int32_t>(blockIdx.x % parts);
  Sum s{-__builtin_inff(), 0.0f};
  const float k = kLog2e / A.r.temperature;
  for (int32_t i = threadIdx.x; i < A.splits; i += 256) join(s, A.part[2 * (row * A.splits + i)], A.part[2 * (row * A.splits + i) + 1], k);
  s = block_sum(s, k);
  const Lse lse = log_sum(s, A.r.temperature);
  if (part == 0 && threadIdx.x == 0) finish(A, row, lse, A.part[2 * A.rows * A.splits + row]);
  if (!A.logprobs) return;
  Part<T> P;
  P.start(A, row, part, A.splits, slots, shared);
  P.write(A.logprobs + row * A.out_stride, lse);
}

// ------------------------------------------------------------------ short rows

// `L` lanes (16 or 64) hold a row: lane i its classes i, i + L, .., E of them.
// What the row's history and biases say of a class is gathered in LDS, in words
// of the row's own that are zero before and after.
template <typename T, int L, int E>
__global__ __launch_bounds__(256) void k_logits_short(LogitArgs A) {
  constexpr int rows = 256 / L;
  __shared__ int32_t count[rows][L * E], place[rows][L * E];
  const int at = threadIdx.x / L, lane = threadIdx.x % L;
  const bool hist = A.r.history_width > 0, biased = A.r.bias_width > 0, own_bias = biased && A.r.bias_per_row;
  const Rules rules(A.r);
  float bias[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    bias[e] = 0.0f;
    count[at][lane + L * e] = place[at][lane + L * e] = 0;
  }
  __syncthreads();
  if (biased && !own_bias) {  // one list for all rows: into registers, once
    for (int i = lane; i < A.r.bias_width; i += L) {
      const int32_t id = A.r.bias_ids[i];
      if (id >= 0 && id < A.classes) atomicMax(&place[at][id], i + 1);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (const int32_t p = place[at][lane + L * e]) bias[e] = A.r.bias_values[p - 1];
  }
  const float k = kLog2e / A.r.temperature;
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows;
  // on their way: the row that follows, its mask, and the number of the mask of the row after it
  float next[E];
  uint32_t next_mask[E];
  int64_t mask_id = -1;
  const auto fetch_id = [&](int64_t row) {
    if (A.r.mask && row < A.rows) mask_id = mask_index(A, row);
  };
  const auto fetch = [&](int64_t row) {
    const T* src = static_cast<const T*>(A.logits) + row * A.stride;
    const bool masked = mask_id >= 0 && mask_id < A.r.mask_rows;
    const uint32_t* mask = A.r.mask + (masked ? mask_id * ((A.classes + 31) / 32) : 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int32_t w = lane + L * e;
      const bool there = row < A.rows && w < A.classes;
      next[e] = there ? as_float(src[w]) : -__builtin_inff();
      next_mask[e] = there && masked ? mask[w >> 5] : 0xFFFFFFFFu;
    }
    fetch_id(row + step);
  };
  fetch_id(static_cast<int64_t>(blockIdx.x) * rows + at);
  fetch(static_cast<int64_t>(blockIdx.x) * rows + at);
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * rows; r0 < A.rows; r0 += step) {
    const int64_t row = r0 + at;
    const bool live = row < A.rows;
    float x[E];
    uint32_t mask[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = next[e], mask[e] = next_mask[e];
    fetch(row + step);
    int32_t n[E];
#pragma unroll
    for (int e = 0; e < E; ++e) n[e] = 0;
    if (hist || own_bias) {
      if (live && hist)
        for (int i = lane; i < A.r.history_width; i += L) {
          const int32_t id = A.r.history[row * A.r.history_width + i];
          if (id >= 0 && id < A.classes) atomicAdd(&count[at][id], 1);
        }
      if (live && own_bias)
        for (int i = lane; i < A.r.bias_width; i += L) {
          const int32_t id = A.r.bias_ids[row * A.r.bias_width + i];
          if (id >= 0 && id < A.classes) atomicMax(&place[at][id], i + 1);
        }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        n[e] = count[at][lane + L * e];
        count[at][lane + L * e] = 0;
        if (own_bias) {
          const int32_t p = place[at][lane + L * e];
          bias[e] = p ? A.r.bias_values[row * A.r.bias_width + p - 1] : 0.0f;
          place[at][lane + L * e] = 0;
        }
      }
      __syncthreads();
    }
    float m = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int32_t w = lane + L * e;
      x[e] = rules(x[e], n[e], bias[e]);
      if (w >= A.classes || !(mask[e] >> (w & 31) & 1u)) x[e] = -__builtin_inff();
      m = fmaxf(m, x[e]);
    }
    Sum s{over_lanes<L>(m, Max()), 0.0f};
    const float base = safe(s.m);
#pragma unroll
    for (int e = 0; e < E; ++e) s.l += term(x[e], base, k);
    s.l = over_lanes<L>(s.l, Plus());
    const Lse lse = log_sum(s, A.r.temperature);
    if (!live) continue;
    if (A.lse && lane == 0) A.lse[row] = lse.value();
    if (A.score) {
      const int32_t t = A.target[row];
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane + L * e == t && t < A.classes) A.score[row] = log_prob(x[e], lse);
      if (lane == 0 && (t < 0 || t >= A.classes)) A.score[row] = t < 0 ? 0.0f : __builtin_nanf("");
    }
    if (A.logprobs) {
      float* dst = A.logprobs + row * A.out_stride;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane + L * e < A.classes) dst[lane + L * e] = log_prob(x[e], lse);
    }
  }
}

template <typename T, int L, int E>
hipError_t run_short(const LogitArgs& A, hipStream_t st) {
  const int64_t groups = (A.rows + 256 / L - 1) / (256 / L);
  // as many workgroups as are resident: each has the next rows on their way while it works on its own
  k_logits_short<T, L, E><<<dim3(static_cast<unsigned>(groups < 2048 ? groups : 2048)), 256, 0, st>>>(A);
  return hipGetLastError();
}

constexpr int kShortClasses = 512;

template <typename T>
hipError_t run(const LogitArgs& A, hipStream_t st) {
  const int32_t C = A.classes;
  if (C <= 16) return run_short<T, 16, 1>(A, st);
  if (C <= 32) return run_short<T, 16, 2>(A, st);
  if (C <= 48) return run_short<T, 16, 3>(A, st);
  if (C <= 64) return run_short<T, 16, 4>(A, st);
  if (C <= 128) return run_short<T, 64, 2>(A, st);
  if (C <= 256) return run_short<T, 64, 4>(A, st);
  if (C <= kShortClasses) return run_short<T, 64, 8>(A, st);
  const int32_t ids = A.r.history_width + A.r.bias_width;
  int32_t slots = 0;
  if (ids)
    for (slots = 64; slots < 2 * ids; slots <<= 1) {
    }
  const size_t per = (C + A.splits - 1) / A.splits + 8;
  const size_t lds = slots || A.r.mask ? ((per + 127) / 128 + 1) * 16 + slots * sizeof(Slot) : 0;
  // a launch has fewer than 2^32 threads
  const int64_t most = (int64_t{1} << 23) / A.splits;
  for (LogitArgs B = A; B.row0 < A.rows; B.row0 += most) {
    const int64_t rows = A.rows - B.row0 < most ? A.rows - B.row0 : most;
    const dim3 grid(static_cast<unsigned>(rows * A.splits));
    if (A.logprobs)
      k_logits<T, false><<<grid, 256, lds, st>>>(B, slots);
    else
      k_logits<T, true><<<grid, 256, lds, st>>>(B, slots);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (A.splits == 1) continue;
    k_logits_join<T><<<dim3(static_cast<unsigned>(A.logprobs ? rows * A.splits : rows)), 256, A.logprobs ? lds : 0, st>>>(B, slots);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

// Parts of a long row: so many that about two workgroups a CU exist, each with
// 1024 classes at least and kPartClasses at most.
int32_t logits_splits(int64_t rows, int32_t classes) {
  if (classes <= kShortClasses) return 1;
  int64_t s = rows > 0 ? (512 + rows - 1) / rows : 1;
  s = s < classes / 1024 ? s : classes / 1024;
  const int64_t least = (classes + kPartClasses - 1) / kPartClasses;
  return static_cast<int32_t>(s < least ? least : s);
}

hipError_t launch_logits(const LogitArgs& A, int dtype, hipStream_t st) {
  return dtype == LB_F32 ? run<float>(A, st) : dtype == LB_BF16 ? run<__bf16>(A, st) : run<_Float16>(A, st);
}

}  // namespace lb
