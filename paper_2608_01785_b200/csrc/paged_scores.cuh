// What the two forms of the paged attention share: a row's view of the keys, and what becomes of a score.
#pragma once
#include "device_ops.h"
#include "ptx.cuh"

namespace hs {
namespace {

// Scores become x in log2 units: x = log2(e) (cap tanh(scale s / cap) - slope |p - j|), or without a cap log2(e) (scale s - ...).
struct ScoreScale {
  float in;        // cap > 0: scale / cap; else scale * log2(e)
  float out;       // cap > 0: cap * log2(e); else 0: not capped
};
inline ScoreScale score_scale(float scale, float cap) {
  const double l2e = 1.4426950408889634074;
  ScoreScale r;
  r.in = cap > 0.f ? float(double(scale) / cap) : float(scale * l2e);
  r.out = cap > 0.f ? float(cap * l2e) : 0.f;
  return r;
}

// tanh to about 1e-7 absolute.  Up to 0.7 in magnitude, where scores that a cap is meant for lie, y P(y^2) with P of degree five fitted to
// tanh(y) / y for the least largest error of y P (4e-9): multiply-adds only, as the unit that takes exponentials has the
// softmax's to do.  Beyond, 1 - 2 / (1 + e^2y).
constexpr float kTanhPoly = 0.7f;
__device__ __forceinline__ float tanh_small(float y) {
  const float u = y * y;
  float p = -0.004874242004007101f;
  p = fmaf(p, u, 0.01973520778119564f);
  p = fmaf(p, u, -0.053383808583021164f);
  p = fmaf(p, u, 0.1332535296678543f);
  p = fmaf(p, u, -0.33332860469818115f);
  p = fmaf(p, u, 0.9999999403953552f);
  return p * y;
}
__device__ __forceinline__ float tanh_any(float y) {
  const float e = fast_exp2(y * 2.8853900817779268f);          // e^2y; infinity gives 1, 0 gives -1
  return fabsf(y) <= kTanhPoly ? tanh_small(y) : 1.f - __fdividef(2.f, 1.f + e);
}

// 16-bit operands of the products: bf16 or fp16.
template <bool F16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (!F16) {
    mma_bf16_16816(d, a, b0, b1);
  } else {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
}
template <bool F16>
__device__ __forceinline__ uint32_t pack_16(float lo, float hi) {
  if constexpr (!F16) {
    return pack_bf16(lo, hi);
  } else {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// Keys of a sequence that a row at position `pos` sees: j < prefix, or from <= j <= pos (from = pos - window + 1, at least 0).
// Rows of one step: the first token row and the number of rows; 0 rows where the step's description is wrong (`error` says how).
struct SeqView {
  int row, rows, kv, prefix, error;
};
__device__ __forceinline__ SeqView view_seq(const hs_paged_attention_t& a, int s) {
  SeqView v;
  v.error = 0;
  v.kv = a.kv_len[s];
  const int most = a.max_pages_per_seq * HS_PAGE_SIZE;
  if (v.kv < 0 || v.kv > most) {
    v.error = kErrBadBlockTable;
    v.kv = v.kv < 0 ? 0 : most;
  }
  if (a.tok_begin) {
    const int b = a.tok_begin[s], e = a.tok_begin[s + 1];
    v.row = b;
    v.rows = e - b;
    if (b < 0 || e < b || e > a.n_tokens || e - b > a.max_q_len) {
      v.error = kErrInvalidArg;
      v.rows = 0;
    }
  } else {
    v.row = s;
    v.rows = 1;
  }
  v.prefix = a.prefix_len ? min(max(a.prefix_len[s], 0), v.kv) : 0;
  return v;
}
// The key pages that the rows at positions p0 .. p1 of a sequence look at: pages 0 .. n_prefix - 1, then first .. first + n - 1.
struct PageRuns {
  int n_prefix, first, n;
  __device__ __forceinline__ int total() const { return n_prefix + n; }
  __device__ __forceinline__ int page(int i) const { return i < n_prefix ? i : first + i - n_prefix; }
};
__device__ __forceinline__ PageRuns page_runs(const SeqView& v, int p0, int p1, int window) {
  PageRuns r;
  r.n_prefix = (v.prefix + 15) >> 4;
  const int from = window > 0 && p0 >= window ? p0 - window + 1 : 0;
  const int end = (min(p1 + 1, v.kv) + 15) >> 4;           // (p1 < 0: no page)
  r.first = max(from >> 4, r.n_prefix);
  r.n = max(end - r.first, 0);
  return r;
}

}  // namespace
}  // namespace hs
