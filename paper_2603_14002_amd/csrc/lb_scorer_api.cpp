// C ABI of the fusion scorer's operators: argument checks and launches.  What
// the device reads (page tables, lengths, ids) is checked by the kernels.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>
#include <exception>
#include <string>

#include "../../include/lightbeam_scorer.h"
#include "lb_scorer.h"

namespace lb {
lb_status set_last_error(lb_status st, const std::string& msg);  // lb_host.cpp
}

using namespace lb;

static_assert(sizeof(lb_kv_cache) == 40, "lb_kv_cache layout");
static_assert(sizeof(lb_kv_batch) == 40, "lb_kv_batch layout");
static_assert(sizeof(lb_rope) == 32, "lb_rope layout");
static_assert(sizeof(lb_logit_rules) == 72, "lb_logit_rules layout");

namespace {

// An argument that the call refuses; caught by `entry`.
struct Refused {
  const char* what;
};

[[noreturn]] void refuse(const char* what) { throw Refused{what}; }
void need(bool ok, const char* what) {
  if (!ok) refuse(what);
}

// Runs an entry point's body: nothing that it throws leaves the library.
template <typename F>
lb_status entry(F&& body) noexcept {
  try {
    try {
      set_last_error(LB_OK, "");
      const hipError_t e = body();
      if (e == hipSuccess) return LB_OK;
      return set_last_error(e == hipErrorOutOfMemory ? LB_ERR_OUT_OF_MEMORY : LB_ERR_HIP, hipGetErrorString(e));
    } catch (const Refused& r) {
      return set_last_error(LB_ERR_INVALID_ARG, r.what);
    }
  } catch (...) {
    return LB_ERR_OUT_OF_MEMORY;
  }
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// a launch has fewer than 2^32 threads: workgroups of 256 threads that a call may need
constexpr int64_t kMostGroups = (1 << 24) - 1;
constexpr float kLog2e = 1.4426950408889634f;

int64_t size_of(int32_t dtype) { return dtype == LB_F32 ? 4 : 2; }

void check_dtype(int32_t dtype) {
  need(dtype == LB_F32 || dtype == LB_BF16 || dtype == LB_F16, "dtype must be LB_F32, LB_BF16 or LB_F16");
}

// a matrix of rows that lanes read or write 16 B at a time
void check_rows(const void* p, int64_t stride, int64_t width, int32_t dtype, int64_t rows, const char* null,
                const char* layout) {
  need(p || rows == 0, null);
  need(aligned(p) && stride >= width && (stride * size_of(dtype)) % 16 == 0 && stride <= (int64_t{1} << 40), layout);
}

// kernels step past the last channel by up to 2048, in 32 bits
void check_widths(int32_t d_in, int32_t d_out) {
  need(d_in >= 8 && d_in % 8 == 0 && d_out >= 8 && d_out % 8 == 0 && d_in <= (1 << 30) && d_out <= (1 << 30),
       "d_in and d_out must be positive multiples of 8, at most 2^30");
}

// whether two matrices of rows have memory in common (true where strides differ and
// their ranges meet)
bool overlap(const void* a, int64_t a_stride, int64_t a_width, const void* b, int64_t b_stride, int64_t b_width, int64_t rows, int64_t size) {
  const __int128 at = reinterpret_cast<uintptr_t>(a), bt = reinterpret_cast<uintptr_t>(b);
  const __int128 a_end = at + (static_cast<__int128>(rows - 1) * a_stride + a_width) * size;
  const __int128 b_end = bt + (static_cast<__int128>(rows - 1) * b_stride + b_width) * size;
  if (a_end <= bt || b_end <= at) return false;
  if (a_stride != b_stride) return true;
  const int64_t line = a_stride * size, from = static_cast<int64_t>(((bt - at) % line + line) % line);  // of b in a's rows
  return from < a_width * size || from + b_width * size > line;
}

KvArgs kv_args(const lb_kv_cache* c, const lb_kv_batch* b, int32_t q_heads) {
  need(c && b, "null descriptor");
  need(c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256, "head_dim must be 64, 128 or 256");
  need(c->kv_heads >= 1 && c->kv_heads <= 1024, "kv_heads must be in 1..1024");
  need(c->page_tokens >= 16 && c->page_tokens <= 256 && (c->page_tokens & (c->page_tokens - 1)) == 0,
       "page_tokens must be 16, 32, 64, 128 or 256");
  need(c->n_pages >= 0 && c->n_pages <= 0x7FFFFFFF, "n_pages out of range");
  need(aligned(c->pages), "pages must be 16-B aligned");
  need((reinterpret_cast<uintptr_t>(c->flags) & 3) == 0, "flags must be 4-B aligned");
  need(b->n_seqs >= 0 && b->n_rows >= 0, "n_seqs and n_rows must not be negative");
  need(b->n_seqs <= (1 << 22) && b->n_rows <= (1 << 24), "n_seqs at most 2^22, n_rows at most 2^24");
  KvArgs a{};
  a.q_heads = q_heads;
  a.kv_heads = c->kv_heads;
  if (b->n_seqs == 0 || b->n_rows == 0) return a;  // nothing to do
  need(c->pages || c->n_pages == 0, "null device pointer: pages");
  need(b->starts && b->lengths && b->pages, "null device pointer in the batch");
  need(b->max_new >= 1, "max_new must be at least 1");
  a.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_tokens));
  need(b->max_pages >= 1 && (static_cast<int64_t>(b->max_pages) << a.page_shift) <= (1 << 30),
       "max_pages must be at least 1, and max_pages * page_tokens at most 2^30");
  a.pages = static_cast<uint8_t*>(c->pages);
  a.n_pages = c->n_pages;
  a.flags = c->flags;
  a.starts = b->starts;
  a.lengths = b->lengths;
  a.table = b->pages;
  a.n_seqs = b->n_seqs;
  a.n_rows = b->n_rows;
  a.max_pages = b->max_pages;
  a.max_new = b->max_new < b->n_rows ? b->max_new : b->n_rows;
  return a;
}

void check_heads(const KvArgs& a) {
  need(a.q_heads >= 1 && a.q_heads % a.kv_heads == 0 && a.q_heads <= 16384,
       "q_heads must be a multiple of kv_heads, at most 16384");
  need(a.n_seqs == 0 || static_cast<int64_t>(a.max_new) * (a.q_heads / a.kv_heads) <= (1 << 30),
       "max_new * q_heads / kv_heads must be at most 2^30");
}

// the plan of a call that launches can take
AttendPlan checked_plan(const KvArgs& a, int32_t head_dim, int32_t dtype) {
  const AttendPlan p = attend_plan(a, head_dim, dtype);
  need(p.groups <= kMostGroups, "too much work for one call: n_seqs or n_rows * q_heads is too large");
  return p;
}

}  // namespace

extern "C" {

lb_status lb_rope_table(int32_t positions, int32_t rot_dim, double base, int32_t scaling, double factor,
                        double trained, double low, double high, float* cos, float* sin) {
  return entry([&] {
    need(positions >= 1 && rot_dim >= 2 && rot_dim % 2 == 0, "positions must be at least 1, rot_dim even and positive");
    need(cos && sin, "null host pointer");
    need(std::isfinite(base) && base > 0, "base must be positive");
    need(scaling == LB_ROPE_PLAIN || scaling == LB_ROPE_LINEAR || scaling == LB_ROPE_BLEND, "unknown scaling");
    need(scaling == LB_ROPE_PLAIN || (std::isfinite(factor) && factor > 0), "factor must be positive");
    need(scaling != LB_ROPE_BLEND || (std::isfinite(trained) && trained > 0 && low > 0 && high > low && std::isfinite(high)),
         "LB_ROPE_BLEND needs trained > 0 and 0 < low < high");
    const int32_t half = rot_dim / 2;
    for (int32_t i = 0; i < half; ++i) {
      double f = std::pow(base, -2.0 * i / rot_dim);
      if (scaling == LB_ROPE_LINEAR) f /= factor;
      if (scaling == LB_ROPE_BLEND) {
        const double turns = trained * f / 6.283185307179586476925;  // trained / wavelength
        double w = (turns - low) / (high - low);
        w = w < 0 ? 0 : w > 1 ? 1 : w;
        f = w * f + (1 - w) * f / factor;
      }
      for (int32_t p = 0; p < positions; ++p) {
        cos[static_cast<int64_t>(p) * half + i] = static_cast<float>(std::cos(p * f));
        sin[static_cast<int64_t>(p) * half + i] = static_cast<float>(std::sin(p * f));
      }
    }
    return hipSuccess;
  });
}

lb_status lb_kv_append(const lb_kv_cache* cache, const lb_kv_batch* batch, const lb_rope* rope, int32_t dtype,
                       int32_t q_heads, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride, void* stream) {
  return entry([&] {
    check_dtype(dtype);
    AppendArgs A{};
    A.kv = kv_args(cache, batch, q_heads);
    need(q_heads >= 0 && q_heads <= 16384, "q_heads must be in 0..16384");
    const int64_t D = cache->head_dim, H = cache->kv_heads, rows = A.kv.n_rows;
    if (rope && rope->rot_dim != 0) {
      need(rope->rot_dim >= 16 && rope->rot_dim % 16 == 0 && rope->rot_dim <= D,
           "rot_dim must be a multiple of 16, at most head_dim");
      need(rope->layout == LB_ROPE_HALF || rope->layout == LB_ROPE_INTERLEAVED, "unknown rotation layout");
      need(rope->positions >= 1 && rope->cos && rope->sin, "the rotation needs cos and sin tables");
      need(aligned(rope->cos) && aligned(rope->sin), "cos and sin must be 16-B aligned");
      A.cos = rope->cos;
      A.sin = rope->sin;
      A.positions = rope->positions;
      A.rot = rope->rot_dim;
      A.interleaved = rope->layout == LB_ROPE_INTERLEAVED;
    }
    check_rows(k, k_stride, H * D, dtype, rows, "null device pointer: k", "k must be 16-B aligned, its row stride at least kv_heads * head_dim and a multiple of 16 B");
    check_rows(v, v_stride, H * D, dtype, rows, "null device pointer: v", "v must be 16-B aligned, its row stride at least kv_heads * head_dim and a multiple of 16 B");
    if (q_heads) {
      check_rows(q, q_stride, q_heads * D, dtype, rows, "null device pointer: q", "q must be 16-B aligned, its row stride at least q_heads * head_dim and a multiple of 16 B");
      check_rows(q_out, q_out_stride, q_heads * D, dtype, rows, "null device pointer: q_out", "q_out must be 16-B aligned, its row stride at least q_heads * head_dim and a multiple of 16 B");
      need(q != q_out || q_stride == q_out_stride, "q_out may be q only with the same row stride");
    }
    A.q = q;
    A.k = k;
    A.v = v;
    A.q_out = q_out;
    A.q_stride = q_stride;
    A.k_stride = k_stride;
    A.v_stride = v_stride;
    A.q_out_stride = q_out_stride;
    return rows == 0 ? hipSuccess : launch_kv_append(A, cache->head_dim, dtype, static_cast<hipStream_t>(stream));
  });
}

lb_status lb_kv_read(const lb_kv_cache* cache, const lb_kv_batch* batch, int32_t dtype, void* k_out,
                     int64_t k_stride, void* v_out, int64_t v_stride, void* stream) {
  return entry([&] {
    check_dtype(dtype);
    ReadArgs A{};
    A.kv = kv_args(cache, batch, 0);
    const int64_t width = static_cast<int64_t>(cache->kv_heads) * cache->head_dim, rows = A.kv.n_rows;
    if (k_out) check_rows(k_out, k_stride, width, dtype, rows, "", "k_out must be 16-B aligned, its row stride at least kv_heads * head_dim and a multiple of 16 B");
    if (v_out) check_rows(v_out, v_stride, width, dtype, rows, "", "v_out must be 16-B aligned, its row stride at least kv_heads * head_dim and a multiple of 16 B");
    A.k = k_out;
    A.v = v_out;
    A.k_stride = k_stride;
    A.v_stride = v_stride;
    if (rows == 0 || (!k_out && !v_out)) return hipSuccess;
    return launch_kv_read(A, cache->head_dim, dtype, static_cast<hipStream_t>(stream));
  });
}

lb_status lb_kv_attend_workspace(const lb_kv_cache* cache, const lb_kv_batch* batch, int32_t q_heads,
                                 int64_t* bytes) {
  return entry([&] {
    need(bytes != nullptr, "null host pointer");
    const KvArgs a = kv_args(cache, batch, q_heads);
    check_heads(a);
    *bytes = a.n_seqs ? checked_plan(a, cache->head_dim, LB_F32).part_floats * 4 : 0;
    return hipSuccess;
  });
}

lb_status lb_kv_attend(const lb_kv_cache* cache, const lb_kv_batch* batch, int32_t dtype, int32_t q_heads,
                       const void* q, int64_t q_stride, float scale, int32_t window, void* out,
                       int64_t out_stride, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  return entry([&] {
    check_dtype(dtype);
    AttendArgs A{};
    A.kv = kv_args(cache, batch, q_heads);
    check_heads(A.kv);
    need(std::isfinite(scale * kLog2e), "scale must be finite");
    need(window >= 0, "window must not be negative");
    const int64_t width = static_cast<int64_t>(q_heads) * cache->head_dim, rows = A.kv.n_rows;
    check_rows(q, q_stride, width, dtype, rows, "null device pointer: q", "q must be 16-B aligned, its row stride at least q_heads * head_dim and a multiple of 16 B");
    check_rows(out, out_stride, width, dtype, rows, "null device pointer: out", "out must be 16-B aligned, its row stride at least q_heads * head_dim and a multiple of 16 B");
    if (rows == 0) return hipSuccess;
    const AttendPlan p = checked_plan(A.kv, cache->head_dim, dtype);
    need(p.part_floats == 0 || (workspace && aligned(workspace) && workspace_bytes >= p.part_floats * 4),
         "the workspace is null, not 16-B aligned or smaller than lb_kv_attend_workspace says");
    A.q = q;
    A.out = out;
    A.q_stride = q_stride;
    A.out_stride = out_stride;
    A.lse = lse;
    A.part = static_cast<float*>(workspace);
    A.scale2 = scale * kLog2e;
    A.window = window < (1 << 30) ? window : 0;  // a sequence has at most 2^30 tokens
    A.tiles = p.tiles;
    A.few_units = static_cast<uint32_t>(p.few_units);
    A.jobs = static_cast<uint32_t>(p.jobs);
    A.splits = p.splits;
    A.part_rows = p.part_rows;
    A.units = p.units;
    A.part_sums = p.part_sums;
    A.few_rows = p.few_rows;
    A.alone = p.alone;
    return launch_kv_attend(A, cache->head_dim, dtype, static_cast<hipStream_t>(stream));
  });
}

lb_status lb_lora_workspace(int64_t rows, int32_t d_in, int32_t d_out, int32_t rank, int64_t* bytes) {
  return entry([&] {
    need(bytes != nullptr, "null host pointer");
    need(rows >= 0 && rows <= (1 << 28), "rows must be in 0..2^28");
    need(rank >= 8 && rank <= 128 && rank % 8 == 0, "rank must be a multiple of 8, at most 128");
    check_widths(d_in, d_out);
    *bytes = lora_whole(rows, d_in, d_out, rank) ? 0 : rows * rank * 4;
    return hipSuccess;
  });
}

lb_status lb_lora_add(int32_t dtype, int64_t rows, int32_t d_in, int32_t d_out, int32_t rank, int32_t n_adapters,
                      const void* x, int64_t x_stride, const void* y, int64_t y_stride, const void* a,
                      const void* b, const int32_t* adapter, const float* scale, void* out, int64_t out_stride,
                      void* workspace, int64_t workspace_bytes, void* stream) {
  return entry([&] {
    check_dtype(dtype);
    need(rows >= 0 && rows <= (1 << 28), "rows must be in 0..2^28");
    need(rank >= 8 && rank <= 128 && rank % 8 == 0, "rank must be a multiple of 8, at most 128");
    check_widths(d_in, d_out);
    need(n_adapters >= 0, "n_adapters must not be negative");
    check_rows(x, x_stride, d_in, dtype, rows, "null device pointer: x", "x must be 16-B aligned, its row stride at least d_in and a multiple of 16 B");
    check_rows(y, y_stride, d_out, dtype, rows, "null device pointer: y", "y must be 16-B aligned, its row stride at least d_out and a multiple of 16 B");
    check_rows(out, out_stride, d_out, dtype, rows, "null device pointer: out", "out must be 16-B aligned, its row stride at least d_out and a multiple of 16 B");
    need(out != y || out_stride == y_stride, "out may be y only with the same row stride");
    need(n_adapters == 0 || (a && b), "null device pointer: a or b");
    need(aligned(a) && aligned(b), "a and b must be 16-B aligned");
    need(adapter || rows == 0, "null device pointer: adapter");
    if (rows == 0) return hipSuccess;
    LoraArgs A{};
    // one launch reads x while other workgroups write out
    A.whole = lora_whole(rows, d_in, d_out, rank) && !overlap(x, x_stride, d_in, out, out_stride, d_out, rows, size_of(dtype));
    need(A.whole || (workspace && aligned(workspace) && workspace_bytes >= rows * rank * 4),
         "the workspace is null, not 16-B aligned or smaller than lb_lora_workspace says (4 * rows * rank bytes where out and x overlap)");
    A.x = x;
    A.y = y;
    A.a = a;
    A.b = b;
    A.out = out;
    A.adapter = adapter;
    A.scale = scale;
    A.h = static_cast<float*>(workspace);
    A.x_stride = x_stride;
    A.y_stride = y_stride;
    A.out_stride = out_stride;
    A.rows = static_cast<int32_t>(rows);
    A.d_in = d_in;
    A.d_out = d_out;
    A.rank = rank;
    A.n_adapters = n_adapters;
    return launch_lora(A, dtype, static_cast<hipStream_t>(stream));
  });
}

lb_status lb_logits_workspace(int64_t rows, int32_t classes, int64_t* bytes) {
  return entry([&] {
    need(bytes != nullptr, "null host pointer");
    need(rows >= 0 && rows <= (1 << 28) && classes >= 1 && classes <= (1 << 30), "rows must be in 0..2^28, classes in 1..2^30");
    const int64_t s = logits_splits(rows, classes);
    *bytes = s > 1 ? (rows * s * 2 + rows) * 4 : 0;
    return hipSuccess;
  });
}

lb_status lb_logits_adjust(int32_t dtype, int64_t rows, int32_t classes, const void* logits,
                           int64_t logits_stride, const lb_logit_rules* rules, const int32_t* target,
                           float* logprobs, int64_t logprobs_stride, float* score, float* lse, void* workspace,
                           int64_t workspace_bytes, void* stream) {
  return entry([&] {
    check_dtype(dtype);
    need(rows >= 0 && rows <= (1 << 28) && classes >= 1 && classes <= (1 << 30), "rows must be in 0..2^28, classes in 1..2^30");
    need(logits || rows == 0, "null device pointer: logits");
    need(logits_stride >= classes && logits_stride <= (int64_t{1} << 40), "logits_stride must be at least classes");
    need(reinterpret_cast<uintptr_t>(logits) % size_of(dtype) == 0, "logits must be aligned to their type");
    need(!logprobs || (logprobs_stride >= classes && logprobs_stride <= (int64_t{1} << 40)), "logprobs_stride must be at least classes");
    need(static_cast<const void*>(logprobs) != logits || !logprobs || (dtype == LB_F32 && logprobs_stride == logits_stride),
         "logprobs may be the logits only where these are LB_F32 with the same stride");
    need(!score || target, "score needs a target");
    LogitArgs A{};
    A.r.temperature = A.r.repetition = 1.0f;
    if (rules) {
      A.r = *rules;
      // their reciprocals have to be numbers too
      need(std::isfinite(A.r.temperature) && A.r.temperature >= FLT_MIN, "temperature must be a normal number above 0");
      need(std::isfinite(A.r.repetition) && A.r.repetition >= FLT_MIN, "repetition must be a normal number above 0");
      need(std::isfinite(A.r.presence) && std::isfinite(A.r.frequency), "presence and frequency must be finite");
      need(A.r.history_width >= 0 && A.r.bias_width >= 0 && A.r.mask_rows >= 0, "widths must not be negative");
      if (!A.r.history) A.r.history_width = 0;
      if (!A.r.bias_ids) A.r.bias_width = 0;
      need(A.r.bias_width == 0 || A.r.bias_values, "bias_ids needs bias_values");
      need(static_cast<int64_t>(A.r.history_width) + A.r.bias_width <= LB_MAX_RULE_IDS, "history_width + bias_width exceeds LB_MAX_RULE_IDS");
      if (!A.r.mask) A.r.mask_rows = 0;
      need(!A.r.mask || A.r.mask_rows >= 1, "mask needs mask_rows");
      need(!A.r.mask || A.r.mask_row || A.r.mask_rows == 1 || A.r.mask_rows >= rows, "without mask_row there must be one mask, or one for each row");
    }
    if (rows == 0) return hipSuccess;
    A.splits = logits_splits(rows, classes);
    need(A.splits == 1 || (workspace && aligned(workspace) && workspace_bytes >= (rows * A.splits * 2 + rows) * 4),
         "the workspace is null, not 16-B aligned or smaller than lb_logits_workspace says");
    A.logits = logits;
    A.stride = logits_stride;
    A.logprobs = logprobs;
    A.out_stride = logprobs_stride;
    A.target = target;
    A.score = score;
    A.lse = lse;
    A.part = static_cast<float*>(workspace);
    A.rows = rows;
    A.classes = classes;
    return launch_logits(A, dtype, static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
