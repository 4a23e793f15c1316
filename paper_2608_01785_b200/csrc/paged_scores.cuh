// What the two forms of the paged attention share: a row's view of the keys, and what becomes of a score.
#pragma once
#include <cfloat>
#include <cmath>

#include "device_ops.h"
#include "ptx.cuh"

namespace hs {
namespace {

// Scores become x in log2 units: x = log2(e) (cap tanh(scale s / cap) - slope |p - j|), or without a cap log2(e) (scale s - ...).
// tanh(y) is y P(y^2) while |y| <= 0.7, with P of degree five fitted to tanh(y) / y for the least largest error of y P (4e-9), or of degree three
// while |y| <= 0.35 (6e-9): multiply-adds only, as the unit that takes exponentials has the softmax's to do.  Scores that a cap is
// meant for lie there.  Beyond, 1 - 2 / (1 + e^2y).  The polynomials stand ready in powers of the raw score, its scale and the cap folded in.
constexpr float kTanhPoly = 0.7f;
struct ScoreScale {
  float in;                // cap > 0: scale / cap; else scale * log2(e)
  float out;               // cap > 0: cap * log2(e); else 0: not capped
  float limit3, limit5;    // largest s^2 of either polynomial; below 0: neither is to be used
  float c3[4], c5[6];      // x = s (c[0] + c[1] s^2 + ..)
};
inline ScoreScale score_scale(float scale, float cap) {
  const double l2e = 1.4426950408889634074;
  const double p3[4] = {0.9999998477158822, -0.3333165701286625, 0.13283323562153154, -0.048376919236770864};
  const double p5[6] = {0.9999999197418465, -0.3333286097994273, 0.13325353247878916, -0.05338380790998526, 0.019735207866603637, -0.00487424220323607};
  ScoreScale r{};
  // (beyond fp32's range the largest number of it: every score but 0 is at the cap then, and 0 stays 0)
  r.in = cap > 0.f ? float(std::fmax(std::fmin(double(scale) / cap, FLT_MAX), -FLT_MAX)) : float(scale * l2e);
  r.out = cap > 0.f ? float(cap * l2e) : 0.f;
  r.limit3 = r.limit5 = -1.f;
  // A polynomial is used where all its coefficients are normal numbers of fp32, so that none is lost: its highest one, out in^7 (or in^11) times p3[3] (p5[5]), is
  // the first to go under where the cap is large for the scale (degree five: scale 1 / 128 with a cap of 100).
  const double in = double(scale) / cap, out = double(cap) * l2e;
  if (cap > 0.f && cap < 1e6f && in > 0.0 && in < 1e2) {
    bool normal3 = true, normal5 = true;
    double f = out * in;
    for (int i = 0; i < 6; ++i, f *= in * in) {
      if (i < 4) {
        r.c3[i] = float(f * p3[i]);
        normal3 = normal3 && std::isnormal(r.c3[i]);
      }
      r.c5[i] = float(f * p5[i]);
      normal5 = normal5 && std::isnormal(r.c5[i]);
    }
    if (normal3) r.limit3 = float(0.35 * 0.35 / (in * in));
    if (normal5) r.limit5 = float(0.7 * 0.7 / (in * in));
  }
  return r;
}

__device__ __forceinline__ float tanh_any(float y) {
  const float e = fast_exp2(y * 2.8853900817779268f);          // e^2y; infinity gives 1, 0 gives -1
  const float u = y * y;
  float p = -0.00487424220323607f;
  p = fmaf(p, u, 0.019735207866603637f);
  p = fmaf(p, u, -0.05338380790998526f);
  p = fmaf(p, u, 0.13325353247878916f);
  p = fmaf(p, u, -0.3333286097994273f);
  p = fmaf(p, u, 0.9999999197418465f);
  return fabsf(y) <= kTanhPoly ? p * y : 1.f - __fdividef(2.f, 1.f + e);
}

// The larger one, or NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Two fp32 at a time.
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(F2 a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
// s (c[0] + c[1] s^2 + ..) + plus
template <int N>
__device__ __forceinline__ F2 odd_poly(F2 s, const float (&c)[N], F2 plus) {
  const F2 u = mul2(s, s);
  F2 p = f2(c[N - 1], c[N - 1]);
#pragma unroll
  for (int i = N - 2; i >= 0; --i) p = fma2(p, u, f2(c[i], c[i]));
  return fma2(p, s, plus);
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
  const int most = row_tokens(a.max_pages_per_seq);
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
