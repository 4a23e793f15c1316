// Rotary positions on q and k together with the scatter of k and v into the paged cache, and the table of cos / sin they use.
//
// Every element is read once and written once; what bounds the kernel is memory, by its latency more than its rate: 8000 rows of 36 heads of 128 in bf16, 152 MB,
// take 31.3 us, 4.9 TB/s.  A unit is sixteen coordinates of one head of one token, two 16-byte pieces of the result: eight pairs that rotate -- (i, i + rot / 2) or
// (2 i, 2 i + 1) -- or sixteen coordinates that are copied.  A warp takes as many whole heads at a time as it has lanes for (four of 128 coordinates), so that its
// loads and stores are runs of 128 bytes and more, and a lane has the same eight pairs in every head: it keeps their 64 bytes of the table until the token changes (read for
// every head, from L1, 34.4 us).  The (token, heads) steps are dealt to the warps in contiguous runs of equal length, whatever the number of tokens.
// Threads of a block x units a lane has on their way, us for 8000 rows of 36 heads of 128 / 1111 rows of 24 of 64 / 64 rows of 36 from fp32: 1024 x 1 34.4 / 4.2 / 5.2,
// 768 x 2 31.7 / 3.5 / 3.9, 640 x 2 31.7 / 3.8 / 3.5, 512 x 2 32.5 / 3.5 / 3.2, 512 x 3 31.6 / 3.7 / 3.2; 640 x 2 is the best of them by a little over nine such sizes.
#include <algorithm>

#include "device_ops.h"
#include "ptx.cuh"

namespace hs {
namespace {

constexpr int RC_THREADS = 640, RT_THREADS = 512;

// Sixteen-byte pieces of eight elements of the source type -> eight floats.
template <int TYPE>
struct Piece;
template <>
struct Piece<HS_TYPE_F32> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    a = f[0];
    b = f[1];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
template <int TYPE>
struct Piece16 {
  uint4 v;
  __device__ __forceinline__ void load(const void* p, int64_t at) { v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (TYPE == HS_TYPE_BF16) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
    }
  }
};
template <>
struct Piece<HS_TYPE_BF16> : Piece16<HS_TYPE_BF16> {};
template <>
struct Piece<HS_TYPE_F16> : Piece16<HS_TYPE_F16> {};

// Eight floats to the cache's type, each rounded to nearest even (beyond fp16's range: infinity, as a conversion of the type has it).
template <bool F16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F16) {
      const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int SRC, bool F16, bool INTERLEAVED>
__global__ void __launch_bounds__(RC_THREADS, 1) rope_cache_kernel(const hs_rope_cache_t a) {
  constexpr int kAhead = SRC == HS_TYPE_F32 ? 1 : 2;          // units a lane has on their way: 64 bytes each from fp32, 32 else
  extern __shared__ uint8_t unused_smem[];
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int per_head = a.head_dim >> 4, heads = 32 / per_head;           // units of a head; heads a warp takes at a time
  const int u = lane % per_head, hg = lane / per_head;
  const int n_heads = a.n_q_heads + 2 * a.n_kv_heads, steps = (n_heads + heads - 1) / heads;
  const bool turns = u < a.rotary_dim >> 4;
  const int lo = !INTERLEAVED && turns ? u * 8 : u * 16, hi = !INTERLEAVED && turns ? lo + (a.rotary_dim >> 1) : lo + 8;
  const int64_t work = int64_t(a.n_tokens) * steps;
  const int64_t warps = int64_t(gridDim.x) * (RC_THREADS / 32), me = int64_t(blockIdx.x) * (RC_THREADS / 32) + (threadIdx.x >> 5);
  int64_t w = work * me / warps;
  const int64_t end = work * (me + 1) / warps;
  int tok = int(w / steps), step = int(w % steps);
  uint16_t* pool = static_cast<uint16_t*>(a.kv_pool) + int64_t(a.layer) * 2 * a.num_pages * a.n_kv_heads * 16 * a.head_dim;
  const int64_t half_pool = int64_t(a.num_pages) * a.n_kv_heads * 16 * a.head_dim;       // K pages, then V pages

  // The lane's eight pairs of the table are the token's, whatever the head: they are fetched when the token changes, with the first rows' loads, as its position is
  // known by then.
  int pos = -1, slot = -1, next_pos = -1, next_slot = -1;
  if (w < end) {
    next_pos = a.tok_pos[tok];
    next_slot = a.tok_slot[tok];
  }
  bool fresh = true, placed = false;
  float4 cs[4];
  while (w < end) {
    Piece<SRC> x[kAhead], y[kAhead];
    int hd[kAhead];
    if (fresh) {
      pos = next_pos;
      slot = next_slot;
      placed = pos >= 0 && pos < a.max_position;
      if (tok + 1 < a.n_tokens) {
        next_pos = a.tok_pos[tok + 1];
        next_slot = a.tok_slot[tok + 1];
      }
      if (turns && placed) {
        const float4* from = reinterpret_cast<const float4*>(a.table + (int64_t(pos) * (a.rotary_dim >> 1) + u * 8) * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) cs[i] = __ldg(from + i);
      }
    }
    const int64_t t = tok;
    fresh = false;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int head = step * heads + hg;
      hd[j] = !fresh && w < end && hg < heads && head < n_heads ? head : -1;
      if (hd[j] >= 0) {
        const void* src;
        int64_t at;
        if (head < a.n_q_heads) {
          src = a.q;
          at = t * a.q_stride + head * a.head_dim;
        } else if (head < a.n_q_heads + a.n_kv_heads) {
          src = a.k;
          at = t * a.k_stride + (head - a.n_q_heads) * a.head_dim;
        } else {
          src = a.v;
          at = t * a.v_stride + (head - a.n_q_heads - a.n_kv_heads) * a.head_dim;
        }
        x[j].load(src, at + lo);
        y[j].load(src, at + hi);
      }
      if (!fresh) {
        ++w;
        if (++step == steps) {                           // the next token's rows are another round's
          step = 0;
          ++tok;
          fresh = true;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (hd[j] < 0) continue;
      const int head = hd[j];
      const bool is_q = head < a.n_q_heads, is_v = head >= a.n_q_heads + a.n_kv_heads;
      float p[8], q[8];
      x[j].get(p);
      y[j].get(q);
      if (turns && !is_v && placed) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {                     // two pairs' (cos, sin)
          if (INTERLEAVED) {
            float (&z)[8] = i < 2 ? p : q;
            rotate_pair(z[4 * (i & 1)], z[4 * (i & 1) + 1], cs[i].x, cs[i].y);
            rotate_pair(z[4 * (i & 1) + 2], z[4 * (i & 1) + 3], cs[i].z, cs[i].w);
          } else {
            rotate_pair(p[2 * i], q[2 * i], cs[i].x, cs[i].y);
            rotate_pair(p[2 * i + 1], q[2 * i + 1], cs[i].z, cs[i].w);
          }
        }
      }
      uint16_t* dst;
      if (is_q) {
        dst = static_cast<uint16_t*>(a.q_out) + t * a.q_out_stride + head * a.head_dim;
        if (!placed) {
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = q[i] = 0.f;
        }
      } else {
        const int page = slot >> 4;
        if (slot < 0 || !placed || page >= a.num_pages) continue;
        const int hk = head - a.n_q_heads - (is_v ? a.n_kv_heads : 0);
        dst = pool + (is_v ? half_pool : 0) + ((int64_t(page) * a.n_kv_heads + hk) * 16 + (slot & 15)) * a.head_dim;
      }
      *reinterpret_cast<uint4*>(dst + lo) = pack8<F16>(p);
      *reinterpret_cast<uint4*>(dst + hi) = pack8<F16>(q);
    }
  }
  // (a row that cannot be placed is reported by one thread of the grid per row)
  for (unsigned t = blockIdx.x * RC_THREADS + threadIdx.x; t < unsigned(a.n_tokens); t += gridDim.x * RC_THREADS) {
    const int p = a.tok_pos[t], s = a.tok_slot[t];
    if (s >= 0 && (p < 0 || p >= a.max_position || (s >> 4) >= a.num_pages)) atomicExch(a.status, kErrInvalidArg);
  }
}

// One thread per (position, pair): sixty-four-bit angle, cos and sin, one rounding.  Made once, so it is left to the 64-bit units: 3.7 us for 4096 positions of 64
// pairs, 12.1 for 32768, 40 for 131072 (67 MB, 1.7 TB/s).
__global__ void __launch_bounds__(RT_THREADS, 1) rope_table_kernel(const hs_rope_table_t a) {
  extern __shared__ double freq[];                        // [rotary_dim / 2]
  griddep_wait();
  const int pairs = a.rotary_dim >> 1;
  for (int i = threadIdx.x; i < pairs; i += RT_THREADS) {
    const double e = -2.0 * i / a.rotary_dim;
    double f = pow(a.base, e);
    if (a.scaling == HS_ROPE_LINEAR) {
      f /= a.factor;
    } else if (a.scaling == HS_ROPE_BASE) {
      f = pow(a.base * pow(a.factor, a.rotary_dim / (a.rotary_dim - 2.0)), e);
    } else if (a.scaling == HS_ROPE_BY_PARTS) {
      const double turns = a.trained_positions * f / 6.283185307179586476925;
      const double keep = fmin(fmax((turns - a.turns_slow) / (a.turns_fast - a.turns_slow), 0.0), 1.0);
      f = f * keep + f / a.factor * (1.0 - keep);
    }
    freq[i] = f;
  }
  __syncthreads();
  const int64_t n = int64_t(a.max_position) * pairs;
  float2* out = reinterpret_cast<float2*>(a.table);
  for (int64_t e = int64_t(blockIdx.x) * RT_THREADS + threadIdx.x; e < n; e += int64_t(gridDim.x) * RT_THREADS) {
    const int64_t p = e / pairs;
    double s, c;
    sincos(double(p) * freq[e - p * pairs], &s, &c);
    out[e] = make_float2(float(c * a.magnitude), float(s * a.magnitude));
  }
}

using RopeKernel = void (*)(hs_rope_cache_t);
template <int SRC>
RopeKernel pick(bool f16, bool interleaved) {
  if (f16) return interleaved ? rope_cache_kernel<SRC, true, true> : rope_cache_kernel<SRC, true, false>;
  return interleaved ? rope_cache_kernel<SRC, false, true> : rope_cache_kernel<SRC, false, false>;
}
RopeKernel pick(int src, bool f16, bool interleaved) {
  return src == HS_TYPE_F32 ? pick<HS_TYPE_F32>(f16, interleaved)
         : src == HS_TYPE_BF16 ? pick<HS_TYPE_BF16>(f16, interleaved) : pick<HS_TYPE_F16>(f16, interleaved);
}

}  // namespace

cudaError_t rope_cache_set_attributes() {
  for (int i = 0; i < 12; ++i) {
    const cudaError_t e = set_kernel_smem(pick(i >> 2, i & 1, i & 2), kMinSmemBytes);
    if (e != cudaSuccess) return e;
  }
  return set_kernel_smem(rope_table_kernel, kMinSmemBytes);
}

cudaError_t launch_rope_cache(const hs_rope_cache_t& a, int sm_budget, cudaStream_t stream) {
  const int heads = 32 / (a.head_dim >> 4), steps = (a.n_q_heads + 2 * a.n_kv_heads + heads - 1) / heads;
  const int64_t blocks = (int64_t(a.n_tokens) * steps + RC_THREADS / 32 - 1) / (RC_THREADS / 32);
  const int grid = int(std::min<int64_t>(blocks, sm_budget));
  return launch_step_kernel(pick(a.src_type, a.cache_type == HS_TYPE_F16, a.interleaved != 0), grid, RC_THREADS, kMinSmemBytes, stream, true, a);
}

cudaError_t launch_rope_table(const hs_rope_table_t& a, int sm_budget, cudaStream_t stream) {
  const int64_t blocks = (int64_t(a.max_position) * (a.rotary_dim >> 1) + RT_THREADS - 1) / RT_THREADS;
  return launch_step_kernel(rope_table_kernel, int(std::min<int64_t>(blocks, sm_budget)), RT_THREADS, kMinSmemBytes, stream, true, a);
}

}  // namespace hs
