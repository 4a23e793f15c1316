// Log probabilities of given tokens, entropy, rank and top alternatives of logit rows, in one pass over the logits.
//
// With k = scale * log2(e), any reference M near max x and d_v = k (x_v - M) (log2 units):
//     s = sum 2^d_v,   t = sum 2^d_v d_v,   logprob_v = ln2 (d_v - log2 s),   entropy = ln2 (log2 s - t / s).
// Every thread keeps (M, s, t) of its own elements and rescales when an element lies 2^10 above its reference; they are joined once per row.
//
// Alternatives.  An element's key orders by value, then by the lower index.  Every thread keeps (a lower bound of) its largest key; the largest
// of them over the sixteen warps, lane by lane, are 32 keys of distinct elements, and the n_top-th largest of those is a bound that no
// alternative lies below.  What reaches the bound is written to a list: about 32 ln(32 / (32 - n_top)) elements of the row reach the final
// one (31 at n_top = 20), and its logarithm of them come while it rises.  The list becomes the alternatives by running top 32 of a warp,
// 32 keys at a time, sorted and merged in the lanes.  A list that overflows is made again from the row itself, by that warp alone: where the first tile of a segment holds
// nothing above -infinity there is no bound behind it, and rows that rise outrun theirs.  us for ordinary rows / all but the last 4096 masked / rising:
// 64 of 152064 fp32, twenty alternatives, 30 / 606 / 1640 (with the events around it); 2047 of 152064 bf16, five, 175 / 25050 / 30200.
//
// Work.  A share, what a block does at a time, is whole rows, one of a row's equal parts, or, in units of 1024 elements, an equal piece of all rows put after one
// another -- the end of a row, whole rows and the beginning of one --, whichever takes its longest share the least time (at the launch).  The block that delivers
// a divided row's last part joins the parts in order.  A share streams through a ring of tiles in shared memory by bulk copies of 16-byte pieces; the
// few elements of a row outside 16-byte boundaries are fetched one by one.
//
// Roles.  Beside the readers one warp requests tiles, one keeps the bound and one ends the rows: a reader that has its part of a row leaves it in shared
// memory, where rows take turns with two places, and goes on with the next row.  The readers wait for one another once in a row, behind its first
// tile, for the first bound.
//
// 2047 rows of 152064 bf16 logits, five alternatives: 162 us, 3.8 TB/s, six tenths of what a copy reaches.  What bounds it is instruction issue: sums and entropy alone take
// 128 us, the alternatives 25, the rank 10.  64 rows of fp32, twenty alternatives: 21.8 us, a row's beginning and end and the join being
// two thirds of it.  Not kept: rings of 4 KB per warp (193 us where this took 173), 8 .. 28 reader warps (180 .. 231), half of the exponentials as polynomials (213),
// a thread's own loop over its candidates (324).
#include <algorithm>

#include "paged_scores.cuh"

namespace hs {
namespace {

constexpr int LP_WARPS = 16, LP_READERS = LP_WARPS * 32, LP_THREADS = LP_READERS + 96;     // and warps that request tiles, keep the bound, end the rows
constexpr int LP_UNIT = 1024;                                                              // elements
constexpr int LP_PIECES = 8, LP_SLOTS = 3;                                                 // 16-byte pieces of a tile per thread; tiles of the ring
constexpr int LP_TILE_BYTES = LP_READERS * LP_PIECES * 16;
constexpr int LP_LIST = 1472;                                                              // candidates of a row
constexpr int LP_MIN_UNITS = 16;                                                           // of a part of a row
constexpr int LP_ROW_COST = 36, LP_JOIN_COST = 54;                                         // units that take as long as a row's beginning and end, as a join
constexpr int LP_JOIN_LOADS = 4;
// A row whose list overflows is looked through by one warp (12 ns an element of a masked bf16 row, 22 of a rising fp32 one) while the others wait for its place: such
// a wait gives up after that much more.
constexpr unsigned long long LP_WAIT_NS = 100;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFar = 1e6f;                                                               // log2 units from zero: fp32 there still has steps of 2^-4
constexpr float kSlack = 10.f;                                                             // log2 units that a logit may lie above its thread's reference

// 16-byte pieces of logits as 32-bit words.  kFloor: what stands for -infinity where its weight is to be 0 and its distance finite; right
// for rows whose maximum lies between kLow and -kLow.
template <int TYPE>
struct Logit;
template <>
struct Logit<HS_TYPE_F32> {
  static constexpr int kSize = 4;
  static constexpr uint32_t kEmpty = 0xff800000u;        // -infinity
  static constexpr float kFloor = -1e36f, kLow = -1e35f;
  static __device__ __forceinline__ void get_above_floor(const uint32_t* w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = max_nan(__uint_as_float(w[i]), kFloor);
  }
  static __device__ __forceinline__ float one(const void* p, int64_t at) { return static_cast<const float*>(p)[at]; }
  static __device__ __forceinline__ void get(const uint32_t* w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ float largest(const uint32_t* w) {
    return max_nan(max_nan(__uint_as_float(w[0]), __uint_as_float(w[1])), max_nan(__uint_as_float(w[2]), __uint_as_float(w[3])));
  }
  static __device__ __forceinline__ float largest_of_all(const uint32_t (&w)[LP_PIECES * 4]) {
    float m[4] = {__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
#pragma unroll
    for (int i = 4; i < LP_PIECES * 4; ++i) m[i & 3] = max_nan(m[i & 3], __uint_as_float(w[i]));
    return max_nan(max_nan(m[0], m[1]), max_nan(m[2], m[3]));
  }
  static __device__ __forceinline__ int above(const uint32_t (&w)[LP_PIECES * 4], float x) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < LP_PIECES * 4; ++i) n += __uint_as_float(w[i]) > x ? 1 : 0;
    return n;
  }
};
template <typename T2>
struct Logit16 {
  static constexpr int kSize = 2;
  static __device__ __forceinline__ T2 two(uint32_t w) { return *reinterpret_cast<const T2*>(&w); }
  static __device__ __forceinline__ float largest(const uint32_t* w) {
    const T2 m = __hmax2_nan(__hmax2_nan(two(w[0]), two(w[1])), __hmax2_nan(two(w[2]), two(w[3])));
    return max_nan(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ float largest_of_all(const uint32_t (&w)[LP_PIECES * 4]) {
    T2 m[4] = {two(w[0]), two(w[1]), two(w[2]), two(w[3])};
#pragma unroll
    for (int i = 4; i < LP_PIECES * 4; ++i) m[i & 3] = __hmax2_nan(m[i & 3], two(w[i]));
    const T2 r = __hmax2_nan(__hmax2_nan(m[0], m[1]), __hmax2_nan(m[2], m[3]));
    return max_nan(__low2float(r), __high2float(r));
  }
  // (whole numbers up to LP_PIECES * 4 per half: exact)
  static __device__ __forceinline__ int count(const uint32_t (&w)[LP_PIECES * 4], T2 t) {
    T2 n[2] = {__hgt2(two(w[0]), t), __hgt2(two(w[1]), t)};
#pragma unroll
    for (int i = 2; i < LP_PIECES * 4; ++i) n[i & 1] = __hadd2(n[i & 1], __hgt2(two(w[i]), t));
    const T2 m = __hadd2(n[0], n[1]);
    return int(__low2float(m) + __high2float(m));
  }
};
template <>
struct Logit<HS_TYPE_BF16> : Logit16<__nv_bfloat162> {
  static constexpr uint32_t kEmpty = 0xff80ff80u;
  static constexpr float kFloor = -1e36f, kLow = -1e35f;
  static __device__ __forceinline__ __nv_bfloat162 floor2() { return __float2bfloat162_rn(kFloor); }
  static __device__ __forceinline__ float one(const void* p, int64_t at) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]); }
  static __device__ __forceinline__ void get(const uint32_t* w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void get_above_floor(const uint32_t* w, float (&x)[8]) {
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto m = __hmax2_nan(two(w[i]), floor2());
      q[i] = *reinterpret_cast<const uint32_t*>(&m);
    }
    get(q, x);
  }
  static __device__ __forceinline__ int above(const uint32_t (&w)[LP_PIECES * 4], float x) { return count(w, __float2bfloat162_rn(x)); }
};
template <>
struct Logit<HS_TYPE_F16> : Logit16<__half2> {
  static constexpr uint32_t kEmpty = 0xfc00fc00u;
  static constexpr float kFloor = -65504.f, kLow = -60000.f;
  static __device__ __forceinline__ __half2 floor2() { return __float2half2_rn(kFloor); }
  static __device__ __forceinline__ float one(const void* p, int64_t at) { return __half2float(static_cast<const __half*>(p)[at]); }
  static __device__ __forceinline__ void get(const uint32_t* w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(two(w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void get_above_floor(const uint32_t* w, float (&x)[8]) {
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto m = __hmax2_nan(two(w[i]), floor2());
      q[i] = *reinterpret_cast<const uint32_t*>(&m);
    }
    get(q, x);
  }
  static __device__ __forceinline__ int above(const uint32_t (&w)[LP_PIECES * 4], float x) { return count(w, __float2half2_rn(x)); }
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
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes),
               "r"(smem_u32(bar))
               : "memory");
}
using Key = unsigned long long;
__device__ __forceinline__ Key larger(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key smaller(Key a, Key b) { return a > b ? b : a; }
// Lanes 0 .. 31 in falling order, from a sequence that rises and falls.
__device__ __forceinline__ Key merge_lanes(Key v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Key w = __shfl_xor_sync(0xffffffffu, v, o);
    v = (lane & o) == 0 ? larger(v, w) : smaller(v, w);
  }
  return v;
}
// How many of the lanes' keys, which are all different, are larger.  (All 32 compared through the warp's scratch: 250 cycles; fifteen exchanges of a sorting
// network took 700.)
__device__ __noinline__ int rank_of(Key k, Key* scratch) {
  scratch[threadIdx.x & 31] = k;
  __syncwarp();
  int n = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const ulonglong2 o = reinterpret_cast<const ulonglong2*>(scratch)[i];
    n += (o.x > k ? 1 : 0) + (o.y > k ? 1 : 0);
  }
  __syncwarp();
  return n;
}
// Empty keys made different from one another, and back.
__device__ __forceinline__ Key distinct(Key k) { return k == 0 ? threadIdx.x & 31 : k; }
__device__ __forceinline__ Key empty_again(Key k) { return k < 32 ? 0 : k; }
// Lanes 0 .. 31 in falling order.
__device__ __forceinline__ Key sort_lanes(Key k, Key* scratch) {
  k = distinct(k);
  const int rank = rank_of(k, scratch);
  scratch[rank] = k;
  __syncwarp();
  k = scratch[threadIdx.x & 31];
  __syncwarp();
  return empty_again(k);
}
// The n-th largest (n = 1 .. 32) of the lanes' keys, in every lane.
__device__ __forceinline__ Key nth_largest(Key k, int n, Key* scratch) {
  k = distinct(k);
  const int rank = rank_of(k, scratch);
  return empty_again(__shfl_sync(0xffffffffu, k, __ffs(__ballot_sync(0xffffffffu, rank == n - 1)) - 1));
}
// The 32 largest of two sets in falling order.
__device__ __forceinline__ Key merge_sorted(Key a, Key b) { return merge_lanes(larger(a, __shfl_sync(0xffffffffu, b, 31 - (threadIdx.x & 31)))); }
// The same with 32 keys in any order, of which a later one than `last` in `a` does not count.
__device__ __noinline__ Key taken(Key a, Key key, Key* scratch) { return merge_sorted(a, sort_lanes(key, scratch)); }
__device__ __forceinline__ void take(Key& a, Key key, int last, Key* scratch) {
  if (__any_sync(0xffffffffu, key > __shfl_sync(0xffffffffu, a, last))) a = taken(a, key, scratch);
}

// What is known of a run of elements: reference M (about the maximum; -infinity: no element above it), s = sum 2^d, t = sum 2^d d with d = k (x - M), elements above the target.
struct Sums {
  float m, s, t;
  int above;
};
// The sums relative to a larger maximum.
__device__ __forceinline__ void raise(Sums& v, float m, float k) {
  if (v.m != m && v.s != 0.f) {                          // (nothing, or weights that are all 0, have no distance)
    const float d = max_nan(k * (v.m - m), -200.f), f = exp2f(d);        // (0 from far below: its product with the distance has to be 0)
    v.t = f * fmaf(v.s, d, v.t);
    v.s *= f;
  }
  v.m = m;
}
// Over the 32 lanes, the same bits in every lane.
__device__ __forceinline__ Sums warp_join(Sums v, float k) {
  raise(v, unordered(__reduce_max_sync(0xffffffffu, ordered(v.m))), k);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
    v.t += __shfl_xor_sync(0xffffffffu, v.t, o);
  }
  v.above = __reduce_add_sync(0xffffffffu, v.above);
  return v;
}

struct Part {                                            // of a divided row, in the workspace
  Sums sums;
  Key keys[HS_MAX_ALTERNATIVES];
};

struct LogprobsParams {
  hs_token_logprobs_t a;
  int shares, units_per_row;
  int parts;                                             // of a row, one a share; 1: whole rows, any number a share; 0: units, cut anywhere
  int base, more;                                        // rows or units of a share; shares with one more, the first ones
  float k;                                               // scale * log2(e)
  unsigned long long wait_ns;                            // after which a wait gives up that may be for the end of a row
};

// What the readers leave of a row for the warp that ends it.
struct RowPlace {
  Key list[LP_LIST];
  Key best[LP_WARPS][32];                                // of each thread; 0: none
  Key bound;
  Sums sums[LP_WARPS];
  float x_t;
  int target, n_list, news;                              // news: best[] has changed since the bound was worked out
};
struct LpSmem {
  uint8_t ring[LP_SLOTS][LP_TILE_BYTES];
  RowPlace place[2];
  uint64_t full[LP_SLOTS], empty[LP_SLOTS], row_full[2], row_empty[2], best_full[2], bound_full[2];
  int abort_flag;
  Key joined[64];                                        // of the parts of a row
  alignas(16) Key scratch[2][32];                        // of the warps that keep the bound and end the rows
};

template <int TYPE>
__global__ void __launch_bounds__(LP_THREADS, 1) token_logprobs_kernel(const __grid_constant__ LogprobsParams p) {
  using L = Logit<TYPE>;
  constexpr int kPer = 16 / L::kSize;                    // elements of a 16-byte piece
  constexpr int kTile = LP_TILE_BYTES / L::kSize;        // and of a tile
  static_assert(kTile % LP_UNIT == 0, "a tile is whole units");
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  LpSmem& sm = *reinterpret_cast<LpSmem*>(smem_raw);
  volatile int* abort_flag = &sm.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int vocab = p.a.vocab, n_top = p.a.n_top, upr = p.units_per_row;
  if (tid == 0) {
    for (int i = 0; i < LP_SLOTS; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], LP_WARPS);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.row_full[i], LP_WARPS);
      mbar_init(&sm.row_empty[i], 1);
      mbar_init(&sm.best_full[i], LP_WARPS);
      mbar_init(&sm.bound_full[i], 1);
      sm.place[i].news = 0;
      sm.place[i].n_list = 0;
    }
    sm.abort_flag = 0;
    fence_barrier_init();
  }
  if (tid < LP_READERS) sm.place[0].best[warp][lane] = sm.place[1].best[warp][lane] = 0;
  __syncthreads();

  // A share is a run of segments: units u0 .. u1 - 1 of a row.  Elements are counted from the 16-byte boundary at or below the row's
  // beginning ("virtual" indices); whole pieces of the row are first .. last - 1.
  auto share_begin = [&](int b) {
    if (p.parts > 1) return b / p.parts * upr + b % p.parts * upr / p.parts;
    return (b * p.base + min(b, p.more)) * (p.parts == 1 ? upr : 1);
  };
  auto share_of = [&](int u) {                           // (of shares that divide rows)
    if (p.parts > 1) return u / upr * p.parts + (u % upr == 0 ? 0 : p.parts - 1);        // (asked of a row's first and last unit)
    const int u_more = p.more * (p.base + 1);
    return u < u_more ? u / (p.base + 1) : p.more + (u - u_more) / p.base;
  };
  struct Segment {
    int row, u0, u1, mis, first, last;
    const char* row_p;
  };
  auto segment_at = [&](int row, int u0, int end) {               // the one that begins with unit u0 of a row, in a share that ends at `end`
    Segment g;
    g.row = row;
    g.u0 = u0;
    g.u1 = min(upr, end - row * upr);
    g.mis = int((reinterpret_cast<uintptr_t>(p.a.logits) / L::kSize + uint64_t(g.row) * uint64_t(p.a.row_stride)) % kPer);
    g.first = g.mis ? kPer : 0;
    g.last = (g.mis + vocab) / kPer * kPer;
    g.row_p = static_cast<const char*>(p.a.logits) + int64_t(g.row) * p.a.row_stride * L::kSize;
    return g;
  };

  // (a wait that gives up lets every role go on to its end, past the waits that follow, without what it waited for)
  bool ok = true;
  if (warp < LP_WARPS) {
    // ------------------------------------------------------------------- the readers
    int slot = 0, at = 0;
    uint32_t phase = 0, row_phase = 0;
    auto target_of = [&](int row) { return row < p.a.n_rows ? p.a.targets[row] : -1; };
    auto target_logit = [&](const char* row_p, int target) { return target >= 0 && target < vocab ? L::one(row_p, target) : INFINITY; };
    // the thread's element outside whole pieces, if it has one: in front of the first one (with unit 0), behind the last one
    auto edge_of = [&](const Segment& g) {
      const int n_front = g.mis && g.u0 == 0 ? min(g.first - g.mis, vocab) : 0;                     // virtual mis .. first - 1
      const int tail = max(g.last, min(g.first, g.mis + vocab)), n_back = g.mis + vocab - tail;      // virtual tail .. mis + vocab - 1
      if (tid < n_front) return tid;
      return tid >= 32 && tid - 32 < n_back && (tail + tid - 32) / LP_UNIT >= g.u0 && (tail + tid - 32) / LP_UNIT < g.u1 ? tail - g.mis + tid - 32 : -1;
    };
    int begin = share_begin(blockIdx.x), end = share_begin(blockIdx.x + 1);
    Segment g0 = segment_at(begin / upr, begin % upr, end);
    int edge = edge_of(g0);
    griddep_wait();                                      // (the divisions do not wait for the kernel in front)
    for (int share = blockIdx.x; share < p.shares;) {
      int row = g0.row, u0 = g0.u0, target = target_of(row);
      float edge_x = edge >= 0 ? L::one(g0.row_p, edge) : 0.f, x_t = target_logit(g0.row_p, target);
      for (; row * upr + u0 < end; ++row, u0 = 0) {
        const Segment g = segment_at(row, u0, end);
        const bool more = (row + 1) * upr < end;  // the share goes on with the next row
        const int next_target = more ? target_of(row + 1) : -1;
        // its target's logit and its elements outside whole pieces are asked for behind this row's first tile: round trips to memory
        float next_x_t = INFINITY, next_edge_x = 0.f;
        int next_edge = -1;
        auto ask_next = [&]() {
          if (!more) return;
          const Segment h = segment_at(row + 1, 0, end);
          next_x_t = target_logit(h.row_p, next_target);
          next_edge = edge_of(h);
          if (next_edge >= 0) next_edge_x = L::one(h.row_p, next_edge);
        };
        const bool count = p.a.rank != nullptr && target >= 0 && target < vocab;
        RowPlace& place = sm.place[at];
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sm.row_empty[at], row_phase ^ 1, abort_flag, p.a.status, p.wait_ns));
        float m = -INFINITY;                             // the thread's reference: its maximum, or up to kSlack below it
        // The distances are k x - (k m rounded to fp32): by this they are too large, all alike, until the row's end takes it out again.  (Of a
        // reference far from zero they are k (x - m).)
        auto slip = [&](float m) {
          const float km = __fmul_rn(m, p.k);
          return fabsf(km) < kFar ? fmaf(m, p.k, -km) : 0.f;
        };
        float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};      // its sums, even and odd elements
        int above = 0;
        auto push = [&](float x, int v) {
          const int i = atomicAdd(&place.n_list, 1);
          if (i < LP_LIST) place.list[i] = make_key(x, v);
        };
        if (edge >= 0) {
          m = edge_x;
          if (edge_x != -INFINITY) {
            const float d = slip(m);
            s[0] = edge_x - edge_x + exp2f(d);           // (NaN of NaN and of infinity)
            t[0] = s[0] * d;
          }
          above = edge_x > x_t ? 1 : 0;
          if (n_top > 0 && edge_x > -INFINITY) push(edge_x, edge);
        }
        for (int v0 = g.u0 * LP_UNIT; v0 < g.u1 * LP_UNIT; v0 += kTile) {
          const bool first = v0 == g.u0 * LP_UNIT;
          const int lo = max(v0, g.first), hi = min(min(v0 + kTile, g.u1 * LP_UNIT), g.last);
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sm.full[slot], phase, abort_flag, p.a.status));
          const int pieces = ok ? max(hi - lo, 0) / kPer : 0;
          const uint8_t* tile = sm.ring[slot];
          uint32_t w[LP_PIECES * 4];
          auto fetch = [&](int i) {
            const uint4 x = *reinterpret_cast<const uint4*>(tile + (i * LP_READERS + tid) * 16);
            w[4 * i] = x.x;
            w[4 * i + 1] = x.y;
            w[4 * i + 2] = x.z;
            w[4 * i + 3] = x.w;
          };
          const bool full = pieces == LP_PIECES * LP_READERS;
          if (full) {
#pragma unroll
            for (int i = 0; i < LP_PIECES; ++i) fetch(i);
          } else {
#pragma unroll
            for (int i = 0; i < LP_PIECES; ++i) {
              w[4 * i] = w[4 * i + 1] = w[4 * i + 2] = w[4 * i + 3] = L::kEmpty;
              if (i * LP_READERS + tid < pieces) fetch(i);
            }
          }
          const float mx = L::largest_of_all(w);
          auto look_for_candidates = [&]() {
            const Key bound = *reinterpret_cast<volatile Key*>(&place.bound);
            const float b_x = bound ? unordered(uint32_t(bound >> 32)) : -INFINITY;
            const int b_v = int(0xffffffffu - unsigned(bound));          // (-1 without a bound: everything above -infinity)
            auto reaches = [&](float x, int v) { return x > b_x || (x == b_x && v <= b_v); };
            // A thread whose largest element reaches the bound has all of its elements looked at by the warp, 32 at a time.  (By itself, in a
            // loop, it held its warp up for 3300 cycles, longer than two tiles take.)
            for (unsigned who = __ballot_sync(0xffffffffu, reaches(mx, lo - g.mis)); who; who &= who - 1) {
              const int of = __ffs(who) - 1;
              const float top = __shfl_sync(0xffffffffu, mx, of);
#pragma unroll 1
              for (int e0 = 0; e0 < LP_PIECES * kPer; e0 += 32) {
                const int e = e0 + lane, i = (e / kPer * LP_READERS + warp * 32 + of) * kPer + e % kPer, v = lo - g.mis + i;
                const float x = e < LP_PIECES * kPer && i < pieces * kPer ? L::one(tile, i) : -INFINITY;
                const bool hit = x > -INFINITY && reaches(x, v);
                const unsigned hits = __ballot_sync(0xffffffffu, hit);
                if (hits == 0) continue;
                const Key key = make_key(x, v);
                const unsigned at_top = __ballot_sync(0xffffffffu, x == top);
                const Key largest = __shfl_sync(0xffffffffu, key, __ffs(at_top | 0x80000000u) - 1);
                int i_list = 0;
                if (lane == 0) {
                  i_list = atomicAdd(&place.n_list, __popc(hits));
                  if (at_top != 0 && largest > place.best[warp][of]) place.best[warp][of] = largest;
                  place.news = 1;
                }
                i_list = __shfl_sync(0xffffffffu, i_list, 0) + __popc(hits & ((1u << lane) - 1u));
                if (hit && i_list < LP_LIST) place.list[i_list] = key;
              }
            }
          };
          auto give_back = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[slot]);
          };
          if (first && n_top > 0) {                      // the first bound is that of all warps: what it needs goes out before the sums
            // (the last index of the thread's first piece, or of its last one, stands for the place of its largest element)
            const int i = L::largest(w) == mx ? 0 : LP_PIECES - 1;
            if (pieces > 0 && mx > -INFINITY) place.best[warp][lane] = make_key(mx, lo - g.mis + (i * LP_READERS + tid) * kPer + kPer - 1);
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.best_full[at]);
          }
          const bool early = !first && full;             // the tile goes back at once, but for the first one, whose bound is on its way, and ragged ones
          if (early) {
            if (n_top > 0) look_for_candidates();
            give_back();
          }
          if (first) ask_next();
          const bool higher = !(mx <= m) && !((mx - m) * p.k <= kSlack);          // (true of the first element above -infinity, and of NaN)
          if (higher) {
            const float to = max_nan(mx, m), d = max_nan(p.k * (m - to) - slip(m) + slip(to), -200.f), f = exp2f(d);      // (nothing so far: s = t = 0)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              t[i] = f * fmaf(s[i], d, t[i]);
              s[i] *= f;
            }
            m = to;
            if (to == INFINITY) s[0] = to - to;          // (a row with infinity has no sum)
          }
          const float from = m == -INFINITY ? 0.f : m, c = -__fmul_rn(from, p.k);
          const bool far = !(fabsf(c) < kFar);
          // one piece after the other: a tile that holds little (a round of pieces takes 390 cycles so, eight take 1200 otherwise), or logits near the
          // type's limits (or NaN), or a scale by which kFloor would not stand for -infinity or leave fp32
          const bool apart = pieces <= 3 * LP_READERS || far || !(from > L::kLow) || p.k > 100.f || p.k < 0.03f;
          if (!apart) {
#pragma unroll
            for (int i = 0; i < LP_PIECES; ++i) {
              float x[kPer];
              L::get_above_floor(w + 4 * i, x);
#pragma unroll
              for (int e = 0; e < kPer; e += 2) {
                const F2 d = fma2(f2(x[e], x[e + 1]), f2(p.k, p.k), f2(c, c));
                float d0, d1;
                split(d, d0, d1);
                const F2 weight = f2(fast_exp2(d0), fast_exp2(d1));
                split(add2(f2(s[0], s[1]), weight), s[0], s[1]);
                split(fma2(weight, d, f2(t[0], t[1])), t[0], t[1]);
              }
            }
          }
          if (apart) {
#pragma unroll 1
            for (int i = 0; i < LP_PIECES && i * LP_READERS + tid < pieces; ++i) {
              // (from memory once more where the tile has gone back)
              const uint4 y = *reinterpret_cast<const uint4*>(early ? reinterpret_cast<const uint8_t*>(g.row_p) + int64_t(lo - g.mis + (i * LP_READERS + tid) * kPer) * L::kSize
                                                                    : tile + (i * LP_READERS + tid) * 16);
              const uint32_t q[4] = {y.x, y.y, y.z, y.w};
              float x[kPer];
              L::get(q, x);
#pragma unroll
              for (int e = 0; e < kPer; ++e) {
                const float d = max_nan(far ? (x[e] - from) * p.k : fmaf(x[e], p.k, c), -126.f), weight = fast_exp2(d);
                s[0] += weight;
                t[0] = fmaf(weight, d, t[0]);
              }
            }
          }
          if (count && !(mx <= x_t)) above += L::above(w, x_t);          // (a maximum that is not a number says nothing about the others)
          if (!early) {
            if (n_top > 0) {
              if (first && ok) ok = __all_sync(0xffffffffu, mbar_wait(&sm.bound_full[at], row_phase, abort_flag, p.a.status));
              look_for_candidates();
            }
            give_back();
          }
          if (++slot == LP_SLOTS) { slot = 0; phase ^= 1; }
        }
        const float e = slip(m), back = exp2f(-e), sum = s[0] + s[1];
        const Sums mine = warp_join(Sums{m, back * sum, back * fmaf(sum, -e, t[0] + t[1]), above}, p.k);
        if (lane == 0) {
          place.sums[warp] = mine;
          if (warp == 0) {
            place.target = target;
            place.x_t = x_t;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.row_full[at]);
        if (++at == 2) { at = 0; row_phase ^= 1; }
        x_t = next_x_t;
        edge = next_edge;
        edge_x = next_edge_x;
        target = next_target;
      }
      share += gridDim.x;
      if (share < p.shares) {
        begin = share_begin(share);
        end = share_begin(share + 1);
        g0 = segment_at(begin / upr, begin % upr, end);
        edge = edge_of(g0);
      }
    }
  } else if (warp == LP_WARPS + 2) {
    // ------------------------------------------------------------ the tiles' requests
    griddep_wait();
    if (lane == 0) {
      int slot = 0;
      uint32_t phase = 0;
      for (int share = blockIdx.x; share < p.shares && ok; share += gridDim.x) {
        const int begin = share_begin(share), end = share_begin(share + 1);
        for (int row = begin / upr, u0 = begin % upr; row * upr + u0 < end && ok; ++row, u0 = 0) {
          const Segment g = segment_at(row, u0, end);
          for (int v = g.u0 * LP_UNIT; v < g.u1 * LP_UNIT; v += kTile) {
            const int lo = max(v, g.first), hi = min(min(v + kTile, g.u1 * LP_UNIT), g.last);
            ok = mbar_wait(&sm.empty[slot], phase ^ 1, abort_flag, p.a.status, p.wait_ns);
            if (!ok) break;
            if (hi > lo) {
              mbar_expect_tx(&sm.full[slot], (hi - lo) * L::kSize);
              bulk_load(sm.ring[slot], g.row_p + int64_t(lo - g.mis) * L::kSize, (hi - lo) * L::kSize, &sm.full[slot]);
            } else {
              mbar_arrive(&sm.full[slot]);
            }
            if (++slot == LP_SLOTS) { slot = 0; phase ^= 1; }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == LP_WARPS) {
    // --------------------------------------------------------------- the bounds of rows
    // The first one of a segment from the first tile's largest keys; then again whenever a reader has found a candidate, until the next segment's
    // largest keys are there.  (This warp alone writes the word, and a bound that comes late finds nobody who reads it.)
    griddep_wait();
    if (n_top > 0) {
      Key* scratch = sm.scratch[0];
      int at = 0;
      uint32_t row_phase = 0;
      for (int share = blockIdx.x; share < p.shares; share += gridDim.x) {
        const int begin = share_begin(share), end = share_begin(share + 1);
        for (int row = begin / upr, u0 = begin % upr; row * upr + u0 < end; ++row, u0 = 0) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sm.best_full[at], row_phase, abort_flag, p.a.status, p.wait_ns));
          RowPlace& place = sm.place[at];
          const int next = at ^ 1;
          const uint32_t next_phase = at ? row_phase ^ 1 : row_phase;
          const bool more = (row + 1) * upr < end || share + int(gridDim.x) < p.shares;
          Key known = 0;
          for (bool first = true;; first = false) {
            if (lane == 0) place.news = 0;
            __syncwarp();
            Key k = 0;
#pragma unroll
            for (int q = 0; q < LP_WARPS; ++q) k = larger(k, reinterpret_cast<volatile Key*>(place.best[q])[lane]);
            const Key bound = nth_largest(k, n_top, scratch);
            if (first || bound > known) {
              known = bound;
              if (lane == 0) *reinterpret_cast<volatile Key*>(&place.bound) = bound;
            }
            __syncwarp();
            if (first && lane == 0) mbar_arrive(&sm.bound_full[at]);
            bool news = false;
            const unsigned long long t0 = globaltimer_ns();
            while (ok && !news && !*abort_flag) {
              if (globaltimer_ns() - t0 > p.wait_ns) {
                *abort_flag = 1;
                atomicExch(p.a.status, kErrTimeout);
              }
              __nanosleep(64);
              if (__any_sync(0xffffffffu, more ? mbar_try_wait(&sm.best_full[next], next_phase) : mbar_try_wait(&sm.row_full[at], row_phase))) break;
              news = __any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&place.news) != 0);
            }
            if (!news) break;
          }
          if (++at == 2) { at = 0; row_phase ^= 1; }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ the rows' ends
    griddep_wait();
    Key* scratch = sm.scratch[1];
    int at = 0;
    uint32_t row_phase = 0;
    int* done_words = reinterpret_cast<int*>(static_cast<char*>(p.a.workspace) + kWsLogprobsDone);
    Part* parts = reinterpret_cast<Part*>(static_cast<char*>(p.a.workspace) + kWsScratch);
    for (int share = blockIdx.x; share < p.shares; share += gridDim.x) {
      const int begin = share_begin(share), end = share_begin(share + 1);
      for (int row = begin / upr, u0 = begin % upr; row * upr + u0 < end; ++row, u0 = 0) {
        const Segment g = segment_at(row, u0, end);
        RowPlace& place = sm.place[at];
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sm.row_full[at], row_phase, abort_flag, p.a.status));
        Sums total = {-INFINITY, 0.f, 0.f, 0};
        if (lane < LP_WARPS) total = place.sums[lane];
        total = warp_join(total, p.k);
        const int target = place.target;
        const float x_t = place.x_t;
        // the alternatives of the segment in falling order, 0 where there are fewer
        Key top = 0;
        if (n_top > 0) {
          const int n_list = ok ? place.n_list : 0;
          const int v_lo = max(g.u0 * LP_UNIT - g.mis, 0), v_hi = min(g.u1 * LP_UNIT - g.mis, vocab);
          if (n_list <= LP_LIST) {
            if (n_list > 64) {
              // candidates of the first, low bounds: those that reach the last one go to the front of the list
              Key k = 0;
#pragma unroll
              for (int q = 0; q < LP_WARPS; ++q) k = larger(k, place.best[q][lane]);
              const Key bound = nth_largest(k, n_top, scratch);
              int kept = 0;
              for (int i = 0; i < n_list; i += 32) {
                const Key c = i + lane < n_list ? place.list[i + lane] : 0;
                const unsigned keep = __ballot_sync(0xffffffffu, c != 0 && c >= bound);
                if (keep >> lane & 1u) place.list[kept + __popc(keep & ((1u << lane) - 1u))] = c;
                kept += __popc(keep);
              }
              __syncwarp();
              for (int i = 0; i < kept; i += 32) take(top, i + lane < kept ? place.list[i + lane] : 0, n_top - 1, scratch);
            } else {
              for (int i = 0; i < n_list; i += 32) take(top, i + lane < n_list ? place.list[i + lane] : 0, n_top - 1, scratch);
            }
            if (n_list < n_top && ok) {                  // fewer than n_top entries above -infinity: the first that are -infinity
              int have = n_list;
              for (int v = v_lo; v < v_hi && have < n_top; v += 32) {
                const bool empty = v + lane < v_hi && L::one(g.row_p, v + lane) == -INFINITY;
                take(top, empty ? make_key(-INFINITY, v + lane) : 0, n_top - 1, scratch);
                have += __popc(__ballot_sync(0xffffffffu, empty));
              }
            }
          } else {
            for (int v = v_lo; v < v_hi; v += 32) take(top, v + lane < v_hi ? make_key(L::one(g.row_p, v + lane), v + lane) : 0, n_top - 1, scratch);
          }
        }
        // the place goes back to the readers
#pragma unroll
        for (int q = 0; q < LP_WARPS; ++q) place.best[q][lane] = 0;
        if (lane == 0) place.n_list = 0;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.row_empty[at]);
        if (++at == 2) { at = 0; row_phase ^= 1; }

        bool whole = g.u1 - g.u0 == upr;
        if (!whole) {
          // a divided row: this share's part, and the join where it is the last one to come
          const int r0 = g.row * upr, r1 = r0 + upr;
          const int f = share_of(r0), l = share_of(r1 - 1);            // shares that hold the row's first and last unit
          Part& part = parts[2 * share + (g.u0 == 0 ? 1 : 0)];         // (the beginning of a row is the share's end)
          if (lane == 0) part.sums = total;
          if (lane < n_top) part.keys[lane] = top;
          __threadfence();
          __syncwarp();
          int n = 0;
          if (lane == 0) n = atomicAdd(done_words + f, 1);
          whole = __shfl_sync(0xffffffffu, n, 0) == l - f;
          if (whole) {
            if (lane == 0) done_words[f] = 0;            // ready for the next call
            __threadfence();
            const int n_parts = l - f + 1;
            auto part_at = [&](int i) -> const Part& { return parts[2 * (f + i) + (i == 0 ? 1 : 0)]; };
            // As with the candidates: a key of each part such that no alternative lies below the n-th largest of them (n parts hold at least n_top keys up
            // to theirs), then what reaches it of all parts' keys, 32 at a time.  What is known from the start is asked for at once.
            const int known = min(n_parts, 32), depth = (n_top + known - 1) / known, n_keys = n_parts * n_top;
            Key c[LP_JOIN_LOADS], k = 0;
            int at_part = n_top > 0 ? lane / n_top : 0, at_key = n_top > 0 ? lane % n_top : 0;
            const int part_step = n_top > 0 ? 32 / n_top : 0, key_step = n_top > 0 ? 32 % n_top : 0;
            auto ask_keys = [&]() {
#pragma unroll
              for (int j = 0; j < LP_JOIN_LOADS; ++j) {
                c[j] = at_part < n_parts ? __ldcg(&part_at(at_part).keys[at_key]) : 0;
                at_part += part_step;
                at_key += key_step;
                if (at_key >= n_top) {
                  at_key -= n_top;
                  ++at_part;
                }
              }
            };
            if (n_top > 0) ask_keys();
            total = Sums{-INFINITY, 0.f, 0.f, 0};
            for (int i = lane; i < n_parts; i += 32) {
              const float4 w = __ldcg(reinterpret_cast<const float4*>(&part_at(i).sums));
              if (n_top > 0) k = larger(k, __ldcg(&part_at(i).keys[depth - 1]));
              Sums v = {w.x, w.y, w.z, __float_as_int(w.w)};
              const float to = max_nan(v.m, total.m);
              raise(v, to, p.k);
              raise(total, to, p.k);
              total.s += v.s;
              total.t += v.t;
              total.above += v.above;
            }
            total = warp_join(total, p.k);
            if (n_top > 0) {
              const Key bound = nth_largest(k, (n_top + depth - 1) / depth, scratch);
              int held = 0;                              // keys that wait in sm.joined
              top = 0;
              for (int i0 = 0;;) {
#pragma unroll
                for (int j = 0; j < LP_JOIN_LOADS; ++j) {
                  const unsigned keep = __ballot_sync(0xffffffffu, c[j] != 0 && c[j] >= bound);
                  if (keep == 0) continue;
                  if (keep >> lane & 1u) sm.joined[held + __popc(keep & ((1u << lane) - 1u))] = c[j];
                  held += __popc(keep);
                  __syncwarp();
                  if (held >= 32) {
                    held -= 32;
                    take(top, sm.joined[held + lane], n_top - 1, scratch);
                  }
                  __syncwarp();
                }
                i0 += 32 * LP_JOIN_LOADS;
                if (i0 >= n_keys) break;
                ask_keys();
              }
              if (held > 0) take(top, lane < held ? sm.joined[lane] : 0, n_top - 1, scratch);
            }
          }
        }
        if (whole) {
          const bool has_target = target >= 0 && target < vocab;
          const float log2_s = log2f(total.s);
          auto logprob = [&](float x) { return total.m == -INFINITY ? -INFINITY : kLn2 * (p.k * (x - total.m) - log2_s); };
          if (lane == 0) {
            p.a.logprob[g.row] = has_target ? logprob(x_t) : 0.f;
            if (p.a.entropy) p.a.entropy[g.row] = total.m == -INFINITY ? 0.f : kLn2 * (log2_s - total.t / total.s);
            if (p.a.rank) p.a.rank[g.row] = has_target ? total.above : -1;
            if (target >= vocab) atomicExch(p.a.status, kErrInvalidArg);
          }
          if (lane < n_top) {
            const int id = top == 0 ? -1 : int(0xffffffffu - unsigned(top));
            p.a.top_ids[int64_t(g.row) * n_top + lane] = id;
            p.a.top_logprobs[int64_t(g.row) * n_top + lane] = top == 0 ? __int_as_float(0x7fc00000) : logprob(unordered(uint32_t(top >> 32)));
          }
        }
      }
    }
  }
  __syncthreads();
  if (*abort_flag) drain_after_abort();
}

constexpr int kLpSmem = int(sizeof(LpSmem)) > kMinSmemBytes ? int(sizeof(LpSmem)) : kMinSmemBytes;
static_assert(kLpSmem <= 227 * 1024, "fits one SM");
static_assert(2 * kMaxShares * sizeof(Part) <= kWsScratchBytes, "two parts per share");
static_assert(kWsLogprobsDone + kMaxShares * 4 <= kWsChunkQueue, "one word per share");

}  // namespace

cudaError_t token_logprobs_set_attributes() {
  cudaError_t e = set_kernel_smem(token_logprobs_kernel<HS_TYPE_F32>, kLpSmem);
  if (e != cudaSuccess) return e;
  if ((e = set_kernel_smem(token_logprobs_kernel<HS_TYPE_BF16>, kLpSmem)) != cudaSuccess) return e;
  return set_kernel_smem(token_logprobs_kernel<HS_TYPE_F16>, kLpSmem);
}

cudaError_t launch_token_logprobs(const hs_token_logprobs_t& a, int sm_count, int sm_budget, cudaStream_t stream) {
  LogprobsParams p{};
  p.a = a;
  const int per = a.type == HS_TYPE_F32 ? 4 : 8;
  p.units_per_row = (a.vocab + per - 1 + LP_UNIT - 1) / LP_UNIT;
  const int units = a.n_rows * p.units_per_row;           // (below 2^31: checked)
  // By what the longest share takes, in units of 1024 elements: whole rows, equal parts of each row, or equal shares that are cut anywhere.  us for whole /
  // parts / anywhere: 41 rows of 23102 fp16 10.2 / - / 21.4; 16 of 152064 fp32 23.2 / 14.1 / 18.3; 64 of 152064 fp32 24.9 / 23.2 / 25.9; 150 of 152064
  // fp32 35.1 / - / 29.1; 2047 of 152064 bf16 160 / - / 165.
  const int most = share_count(sm_count), upr = p.units_per_row;
  const int parts = std::min(most / std::min(a.n_rows, most), upr / LP_MIN_UNITS);
  const int64_t whole = int64_t((a.n_rows + most - 1) / most) * (upr + LP_ROW_COST);
  const int64_t divided = parts > 1 ? (upr + parts - 1) / parts + LP_ROW_COST + LP_JOIN_COST : whole;
  const int64_t anywhere = units / most + (a.n_rows / most + 2) * LP_ROW_COST + LP_JOIN_COST;
  p.parts = whole <= std::min(divided, anywhere) ? 1 : divided <= anywhere ? parts : 0;
  const int pieces = p.parts > 0 ? a.n_rows * p.parts : units;
  p.shares = std::min(most, pieces);
  p.base = pieces / p.shares;
  p.more = pieces % p.shares;
  p.k = float(double(a.scale) * 1.4426950408889634074);
  p.wait_ns = kWaitLimitNs + LP_WAIT_NS * static_cast<unsigned long long>(a.vocab);
  const int grid = std::min(p.shares, sm_budget);
  if (a.type == HS_TYPE_F32) return launch_step_kernel(token_logprobs_kernel<HS_TYPE_F32>, grid, LP_THREADS, kLpSmem, stream, true, p);
  if (a.type == HS_TYPE_BF16) return launch_step_kernel(token_logprobs_kernel<HS_TYPE_BF16>, grid, LP_THREADS, kLpSmem, stream, true, p);
  return launch_step_kernel(token_logprobs_kernel<HS_TYPE_F16>, grid, LP_THREADS, kLpSmem, stream, true, p);
}

}  // namespace hs
