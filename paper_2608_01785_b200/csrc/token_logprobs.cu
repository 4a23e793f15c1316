// Log probabilities of given tokens, entropy, rank and top alternatives of logit rows, in one pass over the logits.
//
// With k = scale * log2(e), M = max x and d_v = k x_v - k M (log2 units, at most 0):
//     s = sum 2^d_v,   t = sum 2^d_v d_v,   logprob_v = ln2 (d_v - log2 s),   entropy = ln2 (log2 s - t / s).
// Every thread keeps (M, s, t) of its own elements and rescales when its maximum moves; they are joined once per row.
//
// Alternatives.  Each lane index keeps the largest value that any of the block's sixteen warps has seen in that lane; the n_top-th
// largest of these 32 values is a value that n_top elements reach at least, so an element below it cannot be an alternative.  Only what reaches it is
// written to a list (about 32 ln(32 / (32 - n_top)) elements of the row reach the final bound, 31 at n_top = 20) and the list is
// sorted by counting at the row's end.  A list that overflows (rows of many equal values) is made again by n_top passes over the row.
//
// Work.  The rows' elements, in units of 1024, are cut into one share per SM of the device, equal and contiguous, whatever the number
// of rows: a share is the end of a row, whole rows and the beginning of one.  The block that delivers a divided row's last
// part joins the parts in order.  A share streams through a ring of tiles in shared memory by bulk copies of 16-byte pieces; the
// few elements of a row outside 16-byte boundaries are fetched one by one.
#include <algorithm>

#include "device_ops.h"
#include "ptx.cuh"

namespace hs {
namespace {

constexpr int LP_WARPS = 16, LP_READERS = LP_WARPS * 32, LP_THREADS = LP_READERS + 32;     // and a warp that requests the tiles
constexpr int LP_UNIT = 1024, LP_TILE = 8 * LP_UNIT, LP_MINE = LP_TILE / LP_READERS;       // elements
constexpr int LP_LIST = kMaxShares * HS_MAX_ALTERNATIVES;                                  // room for a join of all shares' alternatives
constexpr int LP_RING_BYTES = 160 * 1024;
constexpr int LP_MIN_UNITS = 2;                                                            // of a share
constexpr float kLn2 = 0.6931471805599453f;

template <int TYPE>
struct Logit;                                            // one 16-byte piece
template <>
struct Logit<HS_TYPE_F32> {
  static constexpr int kSize = 4;
  static __device__ __forceinline__ float one(const void* p, int64_t at) { return static_cast<const float*>(p)[at]; }
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static constexpr uint32_t kEmpty = 0xff800000u;        // -infinity
};
template <>
struct Logit<HS_TYPE_BF16> {
  static constexpr int kSize = 2;
  static __device__ __forceinline__ float one(const void* p, int64_t at) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]); }
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static constexpr uint32_t kEmpty = 0xff80ff80u;
};
template <>
struct Logit<HS_TYPE_F16> {
  static constexpr int kSize = 2;
  static __device__ __forceinline__ float one(const void* p, int64_t at) { return __half2float(static_cast<const __half*>(p)[at]); }
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static constexpr uint32_t kEmpty = 0xfc00fc00u;
};

// Whole numbers in the order of the floats (and NaN above or below all).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u ^ (u & 0x80000000u ? 0x80000000u : 0xffffffffu)); }
// The larger value is the larger key, and of equal values the lower index.  0 is no key of any element.
__device__ __forceinline__ unsigned long long make_key(float x, int v) {
  return (static_cast<unsigned long long>(ordered(x + 0.f)) << 32) | (0xffffffffu - unsigned(v));       // (-0 counts as 0)
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes),
               "r"(smem_u32(bar))
               : "memory");
}
// The n-th largest (n = 1 .. 32) of the 32 lanes' values, in every lane.
__device__ __forceinline__ uint32_t nth_largest(uint32_t v, int n) {
  const int lane = threadIdx.x & 31;
  int above = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint32_t w = __shfl_sync(0xffffffffu, v, i);
    above += w > v || (w == v && i < lane) ? 1 : 0;
  }
  const unsigned at = __ballot_sync(0xffffffffu, above == n - 1);
  return __shfl_sync(0xffffffffu, v, __ffs(at) - 1);
}

// What is known of a run of elements: maximum (k x, log2 units; -infinity: none), sum, weighted sum, elements above the target.
struct Sums {
  float m, s, t;
  int above;
};
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
  Sums r;
  r.m = max_nan(a.m, b.m);
  r.above = a.above + b.above;
  if (r.m == -INFINITY) {
    r.s = r.t = 0.f;
    return r;
  }
  // (a part without elements has s = t = 0, and its distance, which is infinite, must not meet them)
  const float da = a.s == 0.f ? 0.f : a.m - r.m, db = b.s == 0.f ? 0.f : b.m - r.m;
  const float fa = exp2f(da), fb = exp2f(db);
  r.s = fa * a.s + fb * b.s;
  r.t = fa * fmaf(a.s, da, a.t) + fb * fmaf(b.s, db, b.t);
  return r;
}
__device__ __forceinline__ Sums warp_join(Sums v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Sums w = {__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o), __shfl_xor_sync(0xffffffffu, v.t, o),
                    __shfl_xor_sync(0xffffffffu, v.above, o)};
    const bool low = (threadIdx.x & o) == 0;             // the lower lanes' sums come first in both partners: the same bits
    v = low ? join(v, w) : join(w, v);
  }
  return v;
}

struct Part {                                            // of a divided row, in the workspace
  Sums sums;
  unsigned long long keys[HS_MAX_ALTERNATIVES];
};

struct LogprobsParams {
  hs_token_logprobs_t a;
  int shares, units_per_row;
  float k;                                               // scale * log2(e)
};

template <int TYPE>
struct LpSmem {
  static constexpr int kTileBytes = LP_TILE * Logit<TYPE>::kSize, kSlots = LP_RING_BYTES / kTileBytes;
  uint8_t ring[kSlots][kTileBytes];
  unsigned long long list[LP_LIST];
  unsigned long long top[HS_MAX_ALTERNATIVES];
  uint64_t full[kSlots], empty[kSlots];
  Sums warp_sums[LP_WARPS];
  uint32_t lane_max[2][32];
  Sums row;
  int n_list, abort_flag, flag;
};

template <int TYPE>
__global__ void __launch_bounds__(LP_THREADS, 1) token_logprobs_kernel(const __grid_constant__ LogprobsParams p) {
  using L = Logit<TYPE>;
  using S = LpSmem<TYPE>;
  constexpr int kPer = 16 / L::kSize;                    // elements of a 16-byte piece
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  S& sm = *reinterpret_cast<S*>(smem_raw);
  volatile int* abort_flag = &sm.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int vocab = p.a.vocab, n_top = p.a.n_top, upr = p.units_per_row;
  if (tid == 0) {
    for (int i = 0; i < S::kSlots; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], LP_WARPS);
    }
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (tid < 64) sm.lane_max[tid >> 5][lane] = 0;
  if (tid == 0) sm.n_list = 0;
  __syncthreads();
  griddep_wait();

  const int64_t units = int64_t(p.a.n_rows) * upr;
  int* done_words = reinterpret_cast<int*>(static_cast<char*>(p.a.workspace) + kWsLogprobsDone);
  Part* parts = reinterpret_cast<Part*>(static_cast<char*>(p.a.workspace) + kWsScratch);
  // A share is a run of segments: units u0 .. u1 - 1 of a row.  Elements are counted from the 16-byte boundary at or below the row's
  // beginning ("virtual" indices).
  auto share_begin = [&](int b) { return units * b / p.shares; };
  auto share_of = [&](int64_t u) { return int(((u + 1) * p.shares - 1) / units); };
  auto misaligned = [&](int row) -> int {
    return int((reinterpret_cast<uintptr_t>(p.a.logits) / L::kSize + uint64_t(row) * uint64_t(p.a.row_stride)) % kPer);
  };
  auto row_at = [&](int row) { return static_cast<const char*>(p.a.logits) + int64_t(row) * p.a.row_stride * L::kSize; };

  int slot = 0;
  uint32_t phase = 0;
  if (warp == LP_WARPS) {
    // ------------------------------------------------------------ the tiles' requests
    if (lane == 0) {
      bool ok = true;
      for (int share = blockIdx.x; share < p.shares && ok; share += gridDim.x) {
        const int64_t end = share_begin(share + 1);
        for (int64_t u = share_begin(share); u < end && ok;) {
          const int row = int(u / upr), u0 = int(u - int64_t(row) * upr), u1 = int(std::min<int64_t>(upr, u0 + (end - u)));
          const int mis = misaligned(row);
          // whole pieces of the row: [first, last) in virtual elements
          const int first = mis ? kPer : 0, last = (mis + vocab) / kPer * kPer;
          const char* base = row_at(row) - mis * L::kSize;
          for (int v = u0 * LP_UNIT; v < u1 * LP_UNIT; v += LP_TILE) {
            const int lo = max(v, first), hi = min(min(v + LP_TILE, u1 * LP_UNIT), last);
            ok = mbar_wait(&sm.empty[slot], phase ^ 1, abort_flag, p.a.status);
            if (!ok) break;
            if (hi > lo) {
              mbar_expect_tx(&sm.full[slot], (hi - lo) * L::kSize);
              bulk_load(sm.ring[slot], base + int64_t(lo) * L::kSize, (hi - lo) * L::kSize, &sm.full[slot]);
            } else {
              mbar_arrive(&sm.full[slot]);
            }
            if (++slot == S::kSlots) { slot = 0; phase ^= 1; }
          }
          u += u1 - u0;
        }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------- the readers
    // (a wait that gives up leaves the block's barriers as they are: every warp goes on, without the tiles, to the end)
    bool ok = true;
    int parity = 0;
    for (int share = blockIdx.x; share < p.shares; share += gridDim.x) {
      const int64_t begin = share_begin(share), end = share_begin(share + 1);
      for (int64_t u = begin; u < end;) {
        const int row = int(u / upr), u0 = int(u - int64_t(row) * upr), u1 = int(std::min<int64_t>(upr, u0 + (end - u)));
        const int mis = misaligned(row);
        const int first = mis ? kPer : 0, last = (mis + vocab) / kPer * kPer;
        const char* row_p = row_at(row);
        const int target = p.a.targets[row];
        const bool has_target = target >= 0 && target < vocab;
        const float x_t = has_target ? L::one(row_p, target) : INFINITY;
        Sums my = {-INFINITY, 0.f, 0.f, 0};
        float best = -INFINITY;                          // largest x this thread has seen
        auto push = [&](float x, int v) {
          const int at = atomicAdd(&sm.n_list, 1);
          if (at < LP_LIST) sm.list[at] = make_key(x, v);
        };
        auto add = [&](float x) {                        // x in reach of my.m
          const float d = max_nan(fmaf(x, p.k, my.m == -INFINITY ? 0.f : -my.m), -200.f);
          const float e = fast_exp2(d);
          my.s += e;
          my.t = fmaf(e, d, my.t);
          my.above += x > x_t ? 1 : 0;
        };
        auto raise = [&](float mx) {                     // the thread's maximum becomes mx
          const float m = mx * p.k;
          if (my.s != 0.f) {
            const float dist = my.m - m, f = exp2f(dist);
            my.t = f * fmaf(my.s, dist, my.t);
            my.s *= f;
          }
          my.m = m;
        };
        // the elements outside whole pieces: in front of the first one (with unit 0), behind the last one
        {
          const int n_front = u0 == 0 ? min(first - (mis ? mis : 0), vocab) : 0;                     // virtual mis .. first - 1
          const int tail = max(last, min(first, mis + vocab)), n_back = mis + vocab - tail;            // virtual tail .. mis + vocab - 1
          int v = -1;
          if (tid < n_front) v = tid;
          else if (tid >= 32 && tid - 32 < n_back && (tail + tid - 32) / LP_UNIT >= u0 && (tail + tid - 32) / LP_UNIT < u1) v = tail - mis + tid - 32;
          if (v >= 0) {
            const float x = L::one(row_p, v);
            best = x;
            raise(x);
            add(x);
            if (n_top > 0 && x > -INFINITY) push(x, v);
          }
        }
        bool fresh = true;                               // no tile of the segment read yet
        float bound = -INFINITY;
        for (int v0 = u0 * LP_UNIT; v0 < u1 * LP_UNIT; v0 += LP_TILE) {
          const int lo = max(v0, first), hi = min(min(v0 + LP_TILE, u1 * LP_UNIT), last);
          ok = __all_sync(0xffffffffu, mbar_wait(&sm.full[slot], phase, abort_flag, p.a.status));
          const int pieces = ok ? max(hi - lo, 0) / kPer : 0;
          float x[LP_MINE];
#pragma unroll
          for (int i = 0; i < LP_MINE / kPer; ++i) {
            const int at = i * LP_READERS + tid;
            uint4 w = make_uint4(L::kEmpty, L::kEmpty, L::kEmpty, L::kEmpty);
            if (at < pieces) w = *reinterpret_cast<const uint4*>(sm.ring[slot] + at * 16);
            L::get(w, x + i * kPer);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.empty[slot]);
          if (++slot == S::kSlots) { slot = 0; phase ^= 1; }
          float mx = x[0];
#pragma unroll
          for (int i = 1; i < LP_MINE; ++i) mx = max_nan(mx, x[i]);
          const bool higher = !(mx <= best);
          if (higher) {
            best = max_nan(mx, best);
            raise(best);
          }
#pragma unroll
          for (int i = 0; i < LP_MINE; ++i) add(x[i]);
          if (n_top > 0) {
            if (higher) atomicMax(&sm.lane_max[parity][lane], ordered(best));
            if (fresh) named_barrier_sync(1, LP_READERS);
            bound = unordered(max(nth_largest(reinterpret_cast<volatile uint32_t*>(sm.lane_max[parity])[lane], n_top), ordered(-INFINITY)));
            if (mx >= bound) {
#pragma unroll
              for (int i = 0; i < LP_MINE; ++i)
                if (x[i] >= bound && x[i] > -INFINITY) push(x[i], lo - mis + ((i / kPer) * LP_READERS + tid) * kPer + i % kPer);
            }
          }
          fresh = false;
        }
        my = warp_join(my);
        if (lane == 0) sm.warp_sums[warp] = my;
        named_barrier_sync(1, LP_READERS);
        if (tid < 32) {
          sm.lane_max[parity ^ 1][lane] = 0;
          Sums v = lane < LP_WARPS ? sm.warp_sums[lane] : Sums{-INFINITY, 0.f, 0.f, 0};
          v = warp_join(v);
          if (lane == 0) sm.row = v;
        }
        // the alternatives of the segment: list -> top, sorted; 0 where there are fewer
        const int n_list = sm.n_list;
        auto sort_list = [&](int n) {
          for (int i = tid; i < n; i += LP_READERS) {
            const unsigned long long key = sm.list[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += sm.list[j] > key ? 1 : 0;
            if (rank < n_top) sm.top[rank] = key;
          }
        };
        if (n_top > 0) {
          if (tid < n_top) sm.top[tid] = 0;
          named_barrier_sync(1, LP_READERS);
          const int v_lo = max(u0 * LP_UNIT - mis, 0), v_hi = min(u1 * LP_UNIT - mis, vocab);
          if (n_list <= LP_LIST) {
            sort_list(n_list);
            if (n_list < n_top && warp == 0) {           // fewer than n_top entries above -infinity: the first that are -infinity
              int have = n_list;
              for (int v = v_lo; v < v_hi && have < n_top; v += 32) {
                const bool empty = v + lane < v_hi && L::one(row_p, v + lane) == -INFINITY;
                const unsigned mask = __ballot_sync(0xffffffffu, empty);
                const int at = have + __popc(mask & ((1u << lane) - 1u));
                if (empty && at < n_top) sm.top[at] = make_key(-INFINITY, v + lane);
                have += __popc(mask);
              }
            }
          } else {
            // more candidates than the list holds: the largest key below the last one, n_top times over
            unsigned long long below = ~0ull;
            for (int i = 0; i < n_top; ++i) {
              unsigned long long k = 0;
              for (int v = v_lo + tid; v < v_hi; v += LP_READERS) {
                const unsigned long long c = make_key(L::one(row_p, v), v);
                if (c < below && c > k) k = c;
              }
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) {
                const unsigned long long c = __shfl_xor_sync(0xffffffffu, k, o);
                k = c > k ? c : k;
              }
              if (lane == 0) sm.list[warp] = k;
              named_barrier_sync(1, LP_READERS);
              for (int w = 0; w < LP_WARPS; ++w) k = sm.list[w] > k ? sm.list[w] : k;
              if (tid == 0) sm.top[i] = k;
              below = k;
              named_barrier_sync(1, LP_READERS);
            }
          }
        }
        named_barrier_sync(1, LP_READERS);
        if (tid == 0) sm.n_list = 0;
        bool whole = u1 - u0 == upr;
        if (!whole) {
          // a divided row: this share's part, and the join where it is the last one to come
          const int64_t r0 = int64_t(row) * upr, r1 = r0 + upr;
          const int slot_of = 2 * share + (u0 == 0 ? 1 : 0);           // the beginning of a row is the share's end
          // shares that hold the row's first and last unit
          const int f = share_of(r0), l = share_of(r1 - 1);
          Part& part = parts[slot_of];
          if (tid == 0) part.sums = sm.row;
          if (tid < n_top) part.keys[tid] = sm.top[tid];
          __threadfence();
          named_barrier_sync(1, LP_READERS);
          if (tid == 0) {
            const int n = atomicAdd(done_words + f, 1);
            sm.flag = n == l - f;
            if (n == l - f) done_words[f] = 0;
          }
          named_barrier_sync(1, LP_READERS);
          whole = sm.flag != 0;
          if (whole) {
            __threadfence();
            const int n_parts = l - f + 1;
            auto part_at = [&](int i) -> const Part& { return parts[2 * (f + i) + (i == 0 ? 1 : 0)]; };
            if (warp == 0) {
              Sums v = {-INFINITY, 0.f, 0.f, 0};
              for (int i = lane; i < n_parts; i += 32) {
                const float4 w = __ldcg(reinterpret_cast<const float4*>(&part_at(i).sums));
                v = join(v, Sums{w.x, w.y, w.z, __float_as_int(w.w)});
              }
              v = warp_join(v);
              if (lane == 0) sm.row = v;
            }
            if (n_top > 0) {
              // a part's last key is reached n_top times: what is below the largest of them is no alternative
              unsigned long long least = 0;
              for (int i = lane; i < n_parts; i += 32) {
                const unsigned long long c = __ldcg(&part_at(i).keys[n_top - 1]);
                least = c > least ? c : least;
              }
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) {
                const unsigned long long c = __shfl_xor_sync(0xffffffffu, least, o);
                least = c > least ? c : least;
              }
              for (int i = tid; i < n_parts * n_top; i += LP_READERS) {
                const unsigned long long c = __ldcg(&part_at(i / n_top).keys[i % n_top]);
                if (c >= least && c != 0) sm.list[atomicAdd(&sm.n_list, 1)] = c;
              }
              if (tid < n_top) sm.top[tid] = 0;
              named_barrier_sync(1, LP_READERS);
              sort_list(sm.n_list);
            }
            named_barrier_sync(1, LP_READERS);
            if (tid == 0) sm.n_list = 0;
          }
        }
        if (whole) {
          const Sums v = sm.row;
          const float log2_s = log2f(v.s);
          auto logprob = [&](float x) {
            if (v.m == -INFINITY) return -INFINITY;
            return kLn2 * (fmaf(x, p.k, -v.m) - log2_s);
          };
          if (tid == 0) {
            p.a.logprob[row] = has_target ? logprob(x_t) : 0.f;
            if (p.a.entropy) p.a.entropy[row] = v.m == -INFINITY ? 0.f : kLn2 * (log2_s - v.t / v.s);
            if (p.a.rank) p.a.rank[row] = has_target ? v.above : -1;
            if (target >= vocab) atomicExch(p.a.status, kErrInvalidArg);
          }
          if (tid < n_top) {
            const unsigned long long key = sm.top[tid];
            const int id = key == 0 ? -1 : int(0xffffffffu - unsigned(key));
            p.a.top_ids[int64_t(row) * n_top + tid] = id;
            p.a.top_logprobs[int64_t(row) * n_top + tid] = key == 0 ? __int_as_float(0x7fc00000) : logprob(unordered(uint32_t(key >> 32)));
          }
        }
        named_barrier_sync(1, LP_READERS);               // the row's words are free for the next one
        parity ^= 1;
        u += u1 - u0;
      }
    }
  }
  __syncthreads();
  if (*abort_flag) drain_after_abort();
}

template <int TYPE>
constexpr int lp_smem() {
  return int(sizeof(LpSmem<TYPE>)) > kMinSmemBytes ? int(sizeof(LpSmem<TYPE>)) : kMinSmemBytes;
}
static_assert(lp_smem<HS_TYPE_F32>() <= 227 * 1024 && lp_smem<HS_TYPE_BF16>() <= 227 * 1024, "fits one SM");
static_assert(2 * kMaxShares * sizeof(Part) <= kWsScratchBytes, "two parts per share");
static_assert(kWsLogprobsDone + kMaxShares * 4 <= kWsChunkQueue, "one word per share");

}  // namespace

cudaError_t token_logprobs_set_attributes() {
  cudaError_t e = set_kernel_smem(token_logprobs_kernel<HS_TYPE_F32>, lp_smem<HS_TYPE_F32>());
  if (e != cudaSuccess) return e;
  if ((e = set_kernel_smem(token_logprobs_kernel<HS_TYPE_BF16>, lp_smem<HS_TYPE_BF16>())) != cudaSuccess) return e;
  return set_kernel_smem(token_logprobs_kernel<HS_TYPE_F16>, lp_smem<HS_TYPE_F16>());
}

cudaError_t launch_token_logprobs(const hs_token_logprobs_t& a, int sm_count, int sm_budget, cudaStream_t stream) {
  LogprobsParams p{};
  p.a = a;
  const int per = a.type == HS_TYPE_F32 ? 4 : 8;
  p.units_per_row = (a.vocab + per - 1 + LP_UNIT - 1) / LP_UNIT;
  const int64_t units = int64_t(a.n_rows) * p.units_per_row;
  p.shares = int(std::max<int64_t>(1, std::min<int64_t>(share_count(sm_count), units / LP_MIN_UNITS)));
  p.k = float(double(a.scale) * 1.4426950408889634074);
  const int grid = std::min(p.shares, sm_budget);
  if (a.type == HS_TYPE_F32) return launch_step_kernel(token_logprobs_kernel<HS_TYPE_F32>, grid, LP_THREADS, lp_smem<HS_TYPE_F32>(), stream, true, p);
  if (a.type == HS_TYPE_BF16) return launch_step_kernel(token_logprobs_kernel<HS_TYPE_BF16>, grid, LP_THREADS, lp_smem<HS_TYPE_BF16>(), stream, true, p);
  return launch_step_kernel(token_logprobs_kernel<HS_TYPE_F16>, grid, LP_THREADS, lp_smem<HS_TYPE_F16>(), stream, true, p);
}

}  // namespace hs
