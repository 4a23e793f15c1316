// The best continuations of every request over its beams and the vocabulary, in one pass over the logits.
//
//   row b of a request     L_b = log sum_v exp(scale x_v),   its n_out largest x_v
//   request                the n_out largest  weight_b (S_b + scale x_v - L_b)  of all its beams' largest
//
// Work.  An item is a row or one of its equal parts.  Four teams of four warps share a block, each with an item of its own from a queue, so that one team's
// beginning and end hide behind the others' streams.  A thread reads eight 16-byte pieces of a tile while it works on the last tile's, and keeps
//   M, s        a whole number M near the maximum in log2 units, and s = sum 2^(k x - M), k = scale log2(e): references are changed and joined by exact
//               powers of two.  k is the sum of two fp32 numbers, and a tile's sum is added with its rounding error kept, so that log s is good to 2.5e-6 at worst and 1e-7 as a rule.
//               (A part whose largest logit is 2^20 of those units from zero, as in a row masked with its type's lowest number from end to end, is
//               summed a second time with that logit as its reference.)
//   best, tile  its largest logit, and the first tile that has it; second, with its tile, the largest of its other tiles, third of those that are left.
// At an item's end the n_out-th largest of 64 groups of two threads' (best, tile) bounds its n_out largest logits from below: only threads whose
// own pair reaches it can hold one, a few of 128, and the team looks through that tile's pieces once more, or through the first two tiles', or, where third reaches the bound
// as well, all of a thread's (the L2 has them); it lists what reaches the bound and ranks the list.  The main loop carries no list and no test per element for it.
// The team that delivers a request's last item makes the choice: L_b from the parts, candidates' scores in 64 bits, the same bound, list and ranks.  A list that runs over gives a
// better bound, until only candidates that are all alike are left, which are taken one by one.  It comes behind the team's next item, while the others work on.
//
// 64 requests of 8 beams over 152,064 bf16 logits: 42 us.  The stream ends after 26 of them on average and 30 at most (5.2 TB/s; the exponentials alone would take 20), the items' ends, of 4 us
// each, follow at once where rows are not cut, and a choice takes 4.  Cutting rows in two for a second round that hides the ends costs more than it hides (60 us).  One request of 4 beams: 12.9 us,
// of which the stream is 2: launch, an item's end (2.5), its delivery (2) and the choice (5) are round trips and code that runs once.
#include <float.h>

#include <algorithm>
#include <limits>

#include "paged_scores.cuh"

namespace hs {
namespace {

constexpr int BS_TEAMS = 4, BS_TEAM = 128, BS_THREADS = BS_TEAMS * BS_TEAM, BS_WARPS = BS_TEAM / 32;
constexpr int BS_PIECES = 8, BS_TILE_PIECES = BS_PIECES * BS_TEAM;       // 16-byte pieces of a tile: per thread, in all
constexpr int BS_AHEAD = 2;                                              // tiles that are on their way to L2 before they are loaded (64 x 8 rows, bf16 and fp32: 43.0 and 66.1 us; none 44.6 and 73.3, four 43.7 and 71.5, eight 49.0 and 72.0)
constexpr int BS_LIST = 512;                                             // candidates that a team ranks at a time
constexpr int BS_ITEM_COST = 3;                                          // tiles
constexpr int BS_MAX_PARTS = 64;                                         // of a row
constexpr float BS_FAR = 1048576.f;                                      // log2 units from zero beyond which references are logits
constexpr float BS_SLACK = 16.f;                                         // log2 units that a logit may lie above its thread's reference

using Key = unsigned long long;

struct alignas(16) SelectPart {                          // of a row, in the workspace
  float s_hi, s_lo, m, ref;                              // s_hi + s_lo: sum of 2^(k (x - ref) - m); m is NaN where the part holds NaN or +infinity
  Key keys[HS_MAX_BEAMS];                                // falling; 0: none
};
struct SelectParams {
  hs_beam_select_t a;
  int parts, items;                                      // of a row; of all rows
  int lanes;                                             // the power of two from parts on, at most 32
  double k;                                              // scale log2(e)
  float k_hi, k_lo;                                      // k rounded towards zero, and what that leaves out (above zero)
};
struct alignas(16) SelectTeam {
  Key best[BS_TEAM];
  Key group[64];
  int rank[64];
  Key list[BS_LIST], flat[BS_LIST];
  int token[BS_LIST];
  float score[BS_LIST];
  double sum[BS_WARPS], lse[HS_MAX_BEAMS];
  float m[BS_WARPS], top[BS_WARPS], base[HS_MAX_BEAMS], weight[HS_MAX_BEAMS], ref[HS_MAX_BEAMS];
  int state[HS_MAX_BEAMS];                               // of a beam: 0: no continuation, 1: in use, 2: done
  Key bound;
  int2 flagged[BS_WARPS][64];                            // threads, and a tile that is to be looked at
  int n_list, bad, next, last;
};

// Whole numbers in the order of the floats.  (-0 counts as 0; no NaN comes here.)
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float float_of(uint32_t u) { return __uint_as_float(u ^ (u & 0x80000000u ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ Key order_of(double x) {
  const Key u = Key(__double_as_longlong(x + 0.0));
  return u ^ (u >> 63 ? ~0ull : 1ull << 63);
}
// The larger logit is the larger key, and of equal ones the lower token.
__device__ __forceinline__ Key token_key(float x, int v) { return (Key(order_of(x)) << 32) | (0xffffffffu - unsigned(v)); }
// Candidates of equal rank: the lower beam first, then the larger logit (next to a score that is far from zero the logits' differences vanish in 64 bits, too), then
// the lower place among the beam's candidates, which is the lower token.
constexpr int BS_PLACE_BITS = 11;
__device__ __forceinline__ Key tie_key(int b, Key k, int place) { return (Key(b) << (32 + BS_PLACE_BITS)) | (Key(~uint32_t(k >> 32)) << BS_PLACE_BITS) | unsigned(place); }
__device__ __forceinline__ int beam_of(Key flat) { return int(flat >> (32 + BS_PLACE_BITS)); }
__device__ __forceinline__ int place_of(Key flat) { return int(flat) & ((1 << BS_PLACE_BITS) - 1); }
__device__ __forceinline__ int token_of(Key k) { return int(0xffffffffu - unsigned(k)); }
__device__ __forceinline__ float logit_of(Key k) { return float_of(uint32_t(k >> 32)); }

// In fp32, where a finite number beyond its range is held to its largest: a score of -infinity means no continuation.
__device__ __forceinline__ float held(double x) {
  const float f = float(x);
  return fabsf(f) < INFINITY || fabs(x) == double(INFINITY) || x != x ? f : copysignf(FLT_MAX, f);
}

// The kPer logits of a 16-byte piece.
template <int TYPE>
struct Piece {
  static constexpr int kPer = TYPE == HS_TYPE_F32 ? 4 : 8, kSize = 16 / kPer;
  static __device__ __forceinline__ void get(const uint4& w, float (&x)[kPer]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TYPE == HS_TYPE_F32) {
        x[i] = __uint_as_float(u[i]);
      } else if constexpr (TYPE == HS_TYPE_BF16) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
    }
  }
  static __device__ __forceinline__ float largest(const uint4& w) {          // or NaN
    if constexpr (TYPE == HS_TYPE_F32) {
      return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)), max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
    } else if constexpr (TYPE == HS_TYPE_BF16) {
      const __nv_bfloat162* v = reinterpret_cast<const __nv_bfloat162*>(&w);
      const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(v[0], v[1]), __hmax2_nan(v[2], v[3]));
      return max_nan(__low2float(m), __high2float(m));
    } else {
      const __half2* v = reinterpret_cast<const __half2*>(&w);
      const __half2 m = __hmax2_nan(__hmax2_nan(v[0], v[1]), __hmax2_nan(v[2], v[3]));
      return max_nan(__low2float(m), __high2float(m));
    }
  }
};

// The piece that begins with element e0 of a row whose elements are mis .. end - 1, one by one.
template <int TYPE>
__device__ __noinline__ uint4 edge_piece(const char* base, int e0, int mis, int end) {
  constexpr int kPer = Piece<TYPE>::kPer;
  constexpr uint32_t none = TYPE == HS_TYPE_F32 ? 0xff800000u : TYPE == HS_TYPE_BF16 ? 0xff80ff80u : 0xfc00fc00u;
  uint32_t w[4] = {none, none, none, none};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (e0 + i < mis || e0 + i >= end) continue;
    if constexpr (kPer == 4) {
      w[i] = reinterpret_cast<const uint32_t*>(base)[e0 + i];
    } else {
      const uint32_t h = reinterpret_cast<const uint16_t*>(base)[e0 + i];
      w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | h << 16 : (w[i / 2] & 0xffff0000u) | h;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row as 16-byte pieces, counted from the boundary at or below its beginning: the row is elements mis .. end - 1 of them.
template <int TYPE>
struct Row {
  using P = Piece<TYPE>;
  const char* base;
  int mis, end;
  __device__ __forceinline__ Row(const hs_beam_select_t& a, int row) {
    const char* p = static_cast<const char*>(a.logits) + int64_t(row) * a.row_stride * P::kSize;
    mis = int((reinterpret_cast<uintptr_t>(p) & 15u) / P::kSize);
    base = p - mis * P::kSize;
    end = mis + a.vocab;
  }
  __device__ __forceinline__ int tiles() const { return (end + BS_TILE_PIECES * P::kPer - 1) / (BS_TILE_PIECES * P::kPer); }
  __device__ __forceinline__ uint4 whole(int piece) const {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(base + int64_t(piece) * 16));
    return v;
  }
  // A tile's way from memory to L2, a line a thread.
  __device__ __forceinline__ void ahead(int tile, int tid) const {
    const int piece = tile * BS_TILE_PIECES + tid * (BS_TILE_PIECES / BS_TEAM);
    if (piece * P::kPer < end) asm volatile("prefetch.global.L2 [%0];" ::"l"(base + int64_t(piece) * 16));
  }
  // Any piece: what lies outside the row is -infinity.
  __device__ __forceinline__ uint4 any(int piece) const {
    const int e0 = piece * P::kPer;
    if (e0 >= mis && e0 + P::kPer <= end) return whole(piece);
    constexpr uint32_t none = TYPE == HS_TYPE_F32 ? 0xff800000u : TYPE == HS_TYPE_BF16 ? 0xff80ff80u : 0xfc00fc00u;
    if (e0 >= end || e0 + P::kPer <= mis) return make_uint4(none, none, none, none);
    return edge_piece<TYPE>(base, e0, mis, end);
  }
};

// A warp's part of sum 2^(k (x - ref)) over tiles tile0 .. tile1 - 1, in every lane.  (x - ref is exact where it counts: 32 of k's log2 units are far less than half of
// ref.  A thread adds up to 16 numbers one after the other; from there on the sum is held in 64 bits, as equal addends are rounded to the same side every time.)
template <int TYPE>
__device__ __noinline__ double far_sum(const Row<TYPE>& r, int tile0, int tile1, float ref, float k_hi, float k_lo, int tid) {
  double v = 0.0;
#pragma unroll 1
  for (int tile = tile0; tile < tile1; ++tile) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int i = tile * BS_PIECES; i < (tile + 1) * BS_PIECES; ++i) {
      float x[Piece<TYPE>::kPer];
      Piece<TYPE>::get(r.any(i * BS_TEAM + tid), x);
#pragma unroll
      for (int e = 0; e < Piece<TYPE>::kPer; ++e) {
        const float d = x[e] - ref;
        sum[e & 3] += exp2f(fmaf(d, k_hi, d * k_lo));
      }
    }
    v += double((sum[0] + sum[1]) + (sum[2] + sum[3]));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The n-th largest of 64 groups' keys (each the larger of two threads'), or 0 where fewer groups have one: t.bound, behind the next team_sync.  Called by the whole team
// with a key of each thread.  A thread compares one group with half of the others.
template <typename F>
__device__ __forceinline__ void find_bound(SelectTeam& t, Key mine, int n, int tid, F team_sync) {
  t.best[tid] = mine;
  if (tid < 64) t.rank[tid] = 0;
  if (tid == 0) t.bound = 0;
  team_sync();
  const int i = tid & 63, half = tid >> 6;
  const Key g = max(t.best[i], t.best[i + 64]);
  if (half == 0) t.group[i] = g;
  team_sync();
  int above = 0;
#pragma unroll 4
  for (int j = 32 * half; j < 32 * half + 32; j += 2) {
    const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&t.group[j]);
    above += o.x > g || (o.x == g && j < i) ? 1 : 0;
    above += o.y > g || (o.y == g && j + 1 < i) ? 1 : 0;
  }
  atomicAdd(&t.rank[i], above);
  team_sync();
  if (half == 0 && t.rank[i] == n - 1) t.bound = g;
}

template <int TYPE>
__global__ void __launch_bounds__(BS_THREADS, 1) beam_select_kernel(const __grid_constant__ SelectParams p) {
  using P = Piece<TYPE>;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  const hs_beam_select_t& a = p.a;
  const int team = int(threadIdx.x) / BS_TEAM, tid = int(threadIdx.x) % BS_TEAM, warp = tid >> 5, lane = tid & 31;
  SelectTeam& t = reinterpret_cast<SelectTeam*>(smem_raw)[team];
  auto team_sync = [&]() { named_barrier_sync(1 + team, BS_TEAM); };
  const int n_out = a.n_out;
  int* queue = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsSelectQueue);
  int* done_words = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsSelectDone);
  SelectPart* parts = reinterpret_cast<SelectPart*>(static_cast<char*>(a.workspace) + kWsScratch);
  griddep_wait();

  // Whether an item was a request's last one is known a while after its end: the choice is made behind the item that comes next.
  int item = team * int(gridDim.x) + int(blockIdx.x);    // (the first items on different SMs)
  if (tid == 0) t.last = -1;
#pragma unroll 1
  for (bool more = item < p.items; ; more = item < p.items) {
    const int row = more ? item / p.parts : 0, part_i = item - row * p.parts;
    const bool ended = !more || (a.done != nullptr && a.done[row] != 0);
    if (tid == 0) {
      if (more) t.next = int(gridDim.x) * BS_TEAMS + atomicAdd(queue, 1);
      t.n_list = 0;
      t.bad = 0;
    }
    SelectPart& part = parts[more ? item : 0];
    if (!ended) {
      const Row<TYPE> r(a, row);
      const int tiles = r.tiles(), tile0 = int(int64_t(tiles) * part_i / p.parts), tile1 = int(int64_t(tiles) * (part_i + 1) / p.parts);
      // ------------------------------------------------------------------ the stream
      float m = -INFINITY, s = 0.f, lost = 0.f, best = -INFINITY, second = -INFINITY, third = -INFINITY;   // (of the tiles' largest)
      int best_tile = 0, second_tile = 0, bad = 0;
      auto inside = [&](int tile) {                      // every piece of the tile lies in the row
        return tile * BS_TILE_PIECES * P::kPer >= r.mis && (tile + 1) * BS_TILE_PIECES * P::kPer <= r.end;
      };
      auto load = [&](int tile, uint4 (&w)[BS_PIECES]) {
        if (inside(tile)) {
#pragma unroll
          for (int i = 0; i < BS_PIECES; ++i) w[i] = r.whole(tile * BS_TILE_PIECES + i * BS_TEAM + tid);
        } else {
#pragma unroll
          for (int i = 0; i < BS_PIECES; ++i) w[i] = r.any(tile * BS_TILE_PIECES + i * BS_TEAM + tid);
        }
      };
      uint4 next[BS_PIECES];
      if (tile0 < tile1) load(tile0, next);
#pragma unroll 1
      for (int tile = tile0 + 1; tile < min(tile0 + BS_AHEAD, tile1); ++tile) r.ahead(tile, tid);
#pragma unroll 1
      for (int tile = tile0; tile < tile1; ++tile) {
        uint4 w[BS_PIECES];
#pragma unroll
        for (int i = 0; i < BS_PIECES; ++i) w[i] = next[i];
        if (tile + 1 < tile1) load(tile + 1, next);
        if (tile + BS_AHEAD < tile1) r.ahead(tile + BS_AHEAD, tid);
        float top = P::largest(w[0]);
#pragma unroll
        for (int i = 1; i < BS_PIECES; ++i) top = max_nan(top, P::largest(w[i]));
        if (!(top < INFINITY)) bad = 1;
        if (top > second) {
          third = second;
          const bool first = top > best;
          second = first ? best : top;
          second_tile = first ? best_tile : tile;
        } else {
          third = fmaxf(third, top);
        }
        if (top > best) {
          best = top;
          best_tile = tile;
          const float up = top * p.k_hi;
          if (!(up <= m + BS_SLACK)) {                   // (m is -infinity at first)
            const float to = ceilf(fminf(fmaxf(up, -BS_FAR), BS_FAR));
            if (m > -INFINITY) {
              const float f = exp2f(m - to);             // (whole numbers: exact)
              s *= f;
              lost *= f;
            }
            m = to;
          }
        }
        const float ref = m > -INFINITY ? -m : 0.f;
        const F2 hi2 = f2(p.k_hi, p.k_hi), lo2 = f2(p.k_lo, p.k_lo), ref2 = f2(ref, ref);
        F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < BS_PIECES; ++i) {
          float x[P::kPer];
          P::get(w[i], x);
#pragma unroll
          for (int e = 0; e < P::kPer; e += 2) {
            const F2 x2 = f2(x[e], x[e + 1]);
            float d0, d1;
            split(fma2(x2, lo2, fma2(x2, hi2, ref2)), d0, d1);
            sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], f2(fast_exp2(d0), fast_exp2(d1)));
          }
        }
        float s0, s1;
        split(add2(sum[0], sum[1]), s0, s1);
        const float y = (s0 + s1) - lost, z = s + y;     // (what the addition rounds away is taken from the next one)
        lost = (z - s) - y;
        s = z;
      }
      // ------------------------------------------------------------------ the item's sum, and the bound of its largest
      {
        const float wm = float_of(__reduce_max_sync(0xffffffffu, order_of(m)));
        float v = m > -INFINITY ? s * exp2f(m - wm) : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        const float top = float_of(__reduce_max_sync(0xffffffffu, order_of(best)));
        if (lane == 0) {
          t.m[warp] = wm;
          t.sum[warp] = double(v);
          t.top[warp] = top;
        }
      }
      const Key mine = best > -INFINITY ? (Key(order_of(best)) << 32) | (0xffffffffu - unsigned(best_tile)) : 0ull;
      find_bound(t, mine, n_out, tid, team_sync);
      if (bad) t.bad = 1;
      float top = t.top[0], ref = 0.f;
#pragma unroll
      for (int w = 1; w < BS_WARPS; ++w) top = fmaxf(top, t.top[w]);
      team_sync();
      if (top > -INFINITY && top < INFINITY && !(fabsf(top * p.k_hi) < BS_FAR)) {
        ref = top;
        const double v = far_sum(r, tile0, tile1, ref, p.k_hi, p.k_lo, tid);
        if (lane == 0) {
          t.m[warp] = 0.f;
          t.sum[warp] = v;
        }
      }
      // ------------------------------------------------------------------ what reaches it
      Key least = t.bound;                               // first a (logit, tile), then a key
      bool by_tile = true;
      for (;;) {
        const float least_x = logit_of(least);
        const int least_tile = by_tile && least ? int(0xffffffffu - unsigned(least)) : 0;
        const bool look = mine != 0 && (by_tile ? mine >= least : best >= least_x);
        // pass 0: one or two tiles of the threads that have no more to show; pass 1: all of the others'
        const int tiles_of = !look ? 0 : least == 0 ? 3 : second < least_x ? 1 : third < least_x ? 2 : 3;
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
          const unsigned who = __ballot_sync(0xffffffffu, pass == 0 ? tiles_of == 1 || tiles_of == 2 : tiles_of == 3);
          const unsigned twice = pass == 0 ? __ballot_sync(0xffffffffu, tiles_of == 2) : 0u;
          if (who == 0) continue;
          if (who >> lane & 1u) t.flagged[warp][__popc(who & ((1u << lane) - 1u))] = make_int2(tid, pass == 0 ? best_tile : tile0);
          if (twice >> lane & 1u) t.flagged[warp][__popc(who) + __popc(twice & ((1u << lane) - 1u))] = make_int2(tid, second_tile);
          __syncwarp();
          const int per = pass == 0 ? BS_PIECES : (tile1 - tile0) * BS_PIECES, total = (__popc(who) + __popc(twice)) * per;
#pragma unroll 1
          for (int at = 0; at < total; at += 128) {
            uint4 w[4];
            int piece[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int i = at + 32 * u + lane, f = min(i, total - 1) / per, q = i - f * per;
              const int2 of = t.flagged[warp][f];
              piece[u] = i < total ? (of.y + q / BS_PIECES) * BS_TILE_PIECES + (q % BS_PIECES) * BS_TEAM + of.x : -1;
              if (piece[u] >= 0) w[u] = r.any(piece[u]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              if (piece[u] < 0) continue;
              if (least != 0 && !(P::largest(w[u]) >= least_x)) continue;
              float x[P::kPer];
              P::get(w[u], x);
              const int tile = piece[u] / BS_TILE_PIECES;
#pragma unroll
              for (int e = 0; e < P::kPer; ++e) {
                const Key key = token_key(x[e], piece[u] * P::kPer + e - r.mis);
                const bool in = x[e] > -INFINITY && (least == 0 || (by_tile ? x[e] > least_x || (x[e] == least_x && tile <= least_tile) : key >= least));
                if (in) {
                  const int n = atomicAdd(&t.n_list, 1);
                  if (n < BS_LIST) t.list[n] = key;
                }
              }
            }
          }
          __syncwarp();
        }
        team_sync();
        const int n = t.n_list;
        if (n <= BS_LIST) break;
        // The list has run over: the n_out-th largest of the keys that it holds is a bound that fewer reach.
        for (int i = tid; i < BS_LIST; i += BS_TEAM) {
          int above = 0;
          for (int j = 0; j < BS_LIST; ++j) above += t.list[j] > t.list[i] ? 1 : 0;
          if (above == n_out - 1) t.bound = t.list[i];
        }
        team_sync();
        least = t.bound;
        by_tile = false;
        if (tid == 0) t.n_list = 0;
        team_sync();
      }
      const int n = t.n_list;
      for (int i = tid; i < n; i += BS_TEAM) {
        const Key k = t.list[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) above += t.list[j] > k ? 1 : 0;
        if (above < n_out) part.keys[above] = k;
      }
      if (tid >= n && tid < n_out) part.keys[tid] = 0;
      if (tid == 0) {
        float top = t.m[0];
        for (int w = 1; w < BS_WARPS; ++w) top = fmaxf(top, t.m[w]);
        double sum = 0.0;
        for (int w = 0; w < BS_WARPS; ++w)
          if (t.m[w] > -INFINITY) sum += t.sum[w] * double(exp2f(t.m[w] - top));
        const float hi = float(sum);
        *reinterpret_cast<float4*>(&part) = make_float4(hi, float(sum - double(hi)), t.bad ? NAN : top, ref);
      }
    }
    team_sync();
    const int request = t.last, next = t.next;           // (of the item before, and the one behind this)
    team_sync();
    if (tid == 0) {
      t.last = -1;
      t.n_list = 0;
      if (more) {
        __threadfence();                                 // (of the whole team's part, which the barrier has brought here)
        const int mine = row / a.n_beams, all = a.n_beams * p.parts;
        if (atomicAdd(done_words + mine, 1) == all - 1) {
          done_words[mine] = 0;                          // ready for the next call
          t.last = mine;
          __threadfence();                               // (of the others' parts, for the whole team behind the next barrier)
        }
      }
    }
    if (request >= 0) {
      // -------------------------------------------------------------------- the request's choice
      // Candidates: every part's keys, largest first, a list each.  The first keys that a thread looks at are on their way while the beams' sums are put together.
      const int row0 = request * a.n_beams, n_lists = a.n_beams * p.parts, n_cand = n_lists * n_out, depth = (n_out + n_lists - 1) / n_lists;
      const SelectPart* lists = parts + size_t(row0) * p.parts;
      const bool few = n_cand <= BS_TEAM;                // all of them go into the list
      Key early[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int l = few ? tid / n_out : tid + u * BS_TEAM, k = few ? tid - l * n_out : depth - 1;
        early[u] = l < n_lists && (!few || u == 0) ? __ldcg(&lists[l].keys[k]) : 0;
      }
      // p.lanes lanes a beam: the powers of two of its parts
#pragma unroll 1
      for (int b0 = 0; b0 < a.n_beams; b0 += BS_TEAM / p.lanes) {
        const int b = b0 + tid / p.lanes, at = tid & (p.lanes - 1);
        const bool valid = b < a.n_beams, over = !valid || (a.done != nullptr && a.done[row0 + b] != 0);
        const float base = valid ? a.scores[row0 + b] : 0.f, weight = valid && a.weight ? a.weight[row0 + b] : 1.f;
        double s = 0.0;
        float m = -INFINITY, ref = 0.f;
        int bad = 0, distant = 0;
        float4 q[BS_MAX_PARTS / 32];
#pragma unroll
        for (int u = 0; u < BS_MAX_PARTS / 32; ++u) {
          const int i = at + 32 * u;
          q[u] = !over && i < p.parts ? __ldcg(reinterpret_cast<const float4*>(&lists[b * p.parts + i])) : make_float4(0.f, 0.f, -INFINITY, 0.f);
        }
#pragma unroll
        for (int u = 0; u < BS_MAX_PARTS / 32; ++u) {
          bad |= q[u].z != q[u].z ? 1 : 0;
          distant |= q[u].w != 0.f ? 1 : 0;
          m = fmaxf(m, q[u].z);
        }
        if (__any_sync(0xffffffffu, distant)) {
          // (parts of a row may have different references: how far they are apart is worked out in 64 bits)
          double far = -INFINITY;
          m = -INFINITY;
#pragma unroll
          for (int u = 0; u < BS_MAX_PARTS / 32; ++u) {
            const double f = p.k * double(q[u].w) + double(q[u].z);
            if (f > far) {
              far = f;
              m = q[u].z;
              ref = q[u].w;
            }
          }
#pragma unroll 1
          for (int o = p.lanes >> 1; o > 0; o >>= 1) {
            const double of = __shfl_xor_sync(0xffffffffu, far, o);
            const float om = __shfl_xor_sync(0xffffffffu, m, o), other = __shfl_xor_sync(0xffffffffu, ref, o);
            if (of > far || (of == far && (om > m || (om == m && other > ref)))) {
              far = of;
              m = om;
              ref = other;
            }
          }
        } else {
#pragma unroll 1
          for (int o = p.lanes >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
#pragma unroll
        for (int u = 0; u < BS_MAX_PARTS / 32; ++u) {    // (references of parts near zero are whole numbers: their powers are exact)
          if (q[u].z > -INFINITY) s += (double(q[u].x) + double(q[u].y)) * double(exp2f(float(p.k * (double(q[u].w) - double(ref)) + (double(q[u].z) - double(m)))));
        }
#pragma unroll 1
        for (int o = p.lanes >> 1; o > 0; o >>= 1) {
          s += __shfl_xor_sync(0xffffffffu, s, o);
          bad |= __shfl_xor_sync(0xffffffffu, bad, o);
        }
        if (at == 0 && valid) {
          const double lse = (double(m) + log2(s)) * 0.69314718055994530942;         // and scale ref
          t.lse[b] = lse;
          t.ref[b] = ref;
          t.base[b] = base;
          t.weight[b] = weight;
          t.state[b] = !(weight > 0.f) ? 0 : over ? 2 : bad || m == -INFINITY ? 0 : 1;
          if (a.lse) a.lse[row0 + b] = over ? 0.f : bad ? NAN : m == -INFINITY ? -INFINITY : held(double(a.scale) * double(ref) + lse);
          if (!(weight > 0.f)) atomicExch(a.status, kErrInvalidArg);
        }
      }
      team_sync();
      // A key of beam b: its score, and its rank (0: none).  A beam that is done has one, the first of its first list.
      auto rank_of = [&](int b, bool first, Key k, double& score) {
        score = -INFINITY;
        if (t.state[b] == 2) {
          if (first) score = double(t.base[b]);
        } else if (t.state[b] == 1 && k != 0) {
          score = double(t.base[b]) + (double(a.scale) * (double(logit_of(k)) - double(t.ref[b])) - t.lse[b]);
        }
        const double ranked = double(t.weight[b]) * score;
        return score > -INFINITY && ranked > -INFINITY ? order_of(ranked) : Key(0);
      };
      const int per_beam = p.parts * n_out;              // candidates
      auto append = [&](int b, Key rank, Key k, int c, double score) {
        const int n = atomicAdd(&t.n_list, 1);
        if (n >= BS_LIST) return;
        t.list[n] = rank;
        t.flat[n] = tie_key(b, k, c - b * per_beam);
        t.token[n] = t.state[b] == 2 ? a.end_token : token_of(k);
        t.score[n] = held(score);
      };
      auto candidate = [&](int c, Key& flat, float& score) {             // candidate c of all: its rank, its place among those of equal rank, and score
        const int l = c / n_out, b = l / p.parts;
        const Key k = t.state[b] == 2 ? 0 : __ldcg(&lists[l].keys[c - l * n_out]);
        double s;
        const Key rank = rank_of(b, c == b * per_beam, k, s);
        flat = tie_key(b, k, c - b * per_beam);
        score = held(s);
        return rank;
      };
      if (few) {
        const int b = min(tid / n_out / p.parts, a.n_beams - 1);
        double score;
        const Key k = t.state[b] == 2 ? 0 : early[0], rank = tid < n_cand ? rank_of(b, tid == b * per_beam, k, score) : 0;
        if (rank != 0) append(b, rank, k, tid, score);
        team_sync();
      } else {
        // Every part's keys fall.  With d = n_out / lists (up), each list's d-th key and the n_out / d-th largest (up) of those, there are n_out candidates from that one up:
        // a bound.
        Key top = 0, of[2];
        double score;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int l = tid + u * BS_TEAM, b = min(l / p.parts, a.n_beams - 1);
          of[u] = l < n_lists ? rank_of(b, l == b * p.parts && depth == 1, early[u], score) : 0;
          top = max(top, of[u]);
        }
#pragma unroll 1
        for (int l = tid + 2 * BS_TEAM; l < n_lists; l += BS_TEAM) top = max(top, rank_of(l / p.parts, l % p.parts == 0 && depth == 1, __ldcg(&lists[l].keys[depth - 1]), score));
        find_bound(t, top, (n_out + depth - 1) / depth, tid, team_sync);
        team_sync();
        Key least = t.bound;
        for (;;) {
          // What reaches it: in each list from its first key on until one does not.  A thread takes a list, or, where there are fewer lists than threads, four keys of one.
          const int quarters = n_lists > BS_TEAM ? 1 : (n_out + 3) / 4;
#pragma unroll 1
          for (int u = 0, x = tid; x < n_lists * quarters; ++u, x += BS_TEAM) {
            if (depth == 1 && quarters == 1 && u < 2 && (u == 0 ? of[0] : of[1]) < max(least, Key(1))) continue;
            const int l = x / quarters, b = l / p.parts;
            int k0 = 4 * (x - l * quarters);
            if (t.state[b] != 1) {
              const Key rank = rank_of(b, l == b * p.parts && k0 == 0, 0, score);
              if (rank != 0 && rank >= least) append(b, rank, 0, l * n_out, score);
              continue;
            }
            bool on = true;
#pragma unroll 1
            do {
              Key keys[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) keys[e] = k0 + e < n_out ? __ldcg(&lists[l].keys[k0 + e]) : 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (!on) break;
                const Key rank = rank_of(b, false, keys[e], score);
                on = rank != 0 && rank >= least;
                if (on) append(b, rank, keys[e], l * n_out + k0 + e, score);
              }
              k0 += 4;
            } while (on && quarters == 1 && k0 < n_out);
          }
          team_sync();
          if (t.n_list <= BS_LIST) break;
          // The list has run over.  The n_out-th largest of 64 groups of the ranks that it holds is a bound that fewer reach, unless they are all alike.
          Key mine = 0;
          for (int i = tid; i < BS_LIST; i += BS_TEAM) mine = max(mine, t.list[i]);
          find_bound(t, mine, n_out, tid, team_sync);
          team_sync();
          if (t.bound <= least) break;
          least = t.bound;
          if (tid == 0) t.n_list = 0;
          team_sync();
        }
      }
      int n = t.n_list;
      if (n > BS_LIST) {
        // More ties than the list holds: one continuation after the other, each the best behind the last.
        Key last_rank = ~0ull, last_flat = 0;
        int found = 0;
        for (; found < n_out; ++found) {
          Key rank_b = 0, flat_b = ~0ull;
          float score_b = 0.f;
#pragma unroll 1
          for (int c = tid; c < n_cand; c += BS_TEAM) {
            Key flat;
            float score;
            const Key rank = candidate(c, flat, score);
            if (rank == 0 || rank > last_rank || rank < rank_b) continue;
            if (rank == last_rank && flat <= last_flat) continue;
            if (rank > rank_b || (rank == rank_b && flat < flat_b)) {
              rank_b = rank;
              flat_b = flat;
              score_b = score;
            }
          }
          t.list[tid] = rank_b;                          // (the list's upper half collects what is found)
          t.flat[tid] = flat_b;
          t.score[tid] = score_b;
          team_sync();
          if (warp == 0) {
            int w = lane;
            for (int i = lane + 32; i < BS_TEAM; i += 32)
              if (t.list[i] > t.list[w] || (t.list[i] == t.list[w] && t.flat[i] < t.flat[w])) w = i;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
              const int v = __shfl_xor_sync(0xffffffffu, w, o);
              if (t.list[v] > t.list[w] || (t.list[v] == t.list[w] && (t.flat[v] < t.flat[w] || (t.flat[v] == t.flat[w] && v < w)))) w = v;
            }
            if (lane == 0) {
              t.list[BS_TEAM + found] = t.list[w];
              t.flat[BS_TEAM + found] = t.flat[w];
              t.score[BS_TEAM + found] = t.score[w];
            }
          }
          team_sync();
          last_rank = t.list[BS_TEAM + found];
          last_flat = t.flat[BS_TEAM + found];
          if (last_rank == 0) break;
        }
        if (tid < found) {
          t.list[tid] = t.list[BS_TEAM + tid];
          const Key f = t.flat[BS_TEAM + tid];
          const int b = beam_of(f), c = place_of(f), in_list = c / n_out;
          t.flat[tid] = f;
          t.score[tid] = t.score[BS_TEAM + tid];
          t.token[tid] = t.state[b] == 2 ? a.end_token : token_of(__ldcg(&lists[b * p.parts + in_list].keys[c - in_list * n_out]));
        }
        n = found;
        team_sync();
      }
      auto put = [&](int place, float score, int parent, int token, int over) {
        const int64_t at = int64_t(request) * n_out + place;
        a.out_score[at] = score;
        a.out_parent[at] = parent;
        a.out_token[at] = token;
        if (a.out_done) a.out_done[at] = over;
      };
      for (int i = tid; i < n; i += BS_TEAM) {
        const Key k = t.list[i], f = t.flat[i];
        int above = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) {                    // (both numbers are read in any case: no answer is waited for before the next is asked for)
          const Key r = t.list[j], g = t.flat[j];
          above += int(r > k) | (int(r == k) & int(g < f));
        }
        if (above >= n_out) continue;
        const int b = beam_of(f), token = t.token[i];
        put(above, t.score[i], row0 + b, token, t.state[b] == 2 || token == a.end_token ? 1 : 0);
      }
      if (tid >= n && tid < n_out) put(tid, -INFINITY, -1, -1, 0);
      team_sync();                                       // (everybody has read what the next item writes over)
    }
    if (!more) {
      team_sync();
      if (request < 0 && t.last < 0) break;
    }
    if (more) item = next;
  }
  __syncthreads();
  // the last block to leave puts the queue back to zero
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(queue + 1, 1) == int(gridDim.x) - 1) {
      queue[0] = 0;
      queue[1] = 0;
    }
  }
}

constexpr int kSelectSmem = BS_TEAMS * int(sizeof(SelectTeam)) > kMinSmemBytes ? BS_TEAMS * int(sizeof(SelectTeam)) : kMinSmemBytes;
static_assert(sizeof(SelectTeam) % 16 == 0 && kSelectSmem <= 227 * 1024, "fits one SM");
static_assert(BS_MAX_PARTS * HS_MAX_BEAMS <= 1 << BS_PLACE_BITS, "a beam's candidates");
static_assert(BS_LIST >= BS_TEAM + HS_MAX_BEAMS, "the list's upper half holds the continuations");
constexpr int64_t kMaxRows = 65536;
static_assert(kMaxRows * sizeof(SelectPart) <= kWsScratchBytes, "a part per row");
static_assert(kWsSelectQueue + 8 <= kWsSelectDone && kWsSelectDone + HS_DEVICE_MAX_SEQS * 4 <= kWsSharedQueue, "one word per request");

using SelectKernel = void (*)(SelectParams);
SelectKernel pick(int type) {
  return type == HS_TYPE_F32 ? beam_select_kernel<HS_TYPE_F32> : type == HS_TYPE_BF16 ? beam_select_kernel<HS_TYPE_BF16> : beam_select_kernel<HS_TYPE_F16>;
}

}  // namespace

cudaError_t beam_select_set_attributes() {
  for (int type = HS_TYPE_F32; type <= HS_TYPE_F16; ++type) {
    const cudaError_t e = set_kernel_smem(pick(type), kSelectSmem);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_beam_select(const hs_beam_select_t& a, int sm_count, int sm_budget, cudaStream_t stream) {
  SelectParams p{};
  p.a = a;
  const double k = p.k = double(a.scale) * 1.4426950408889634074;
  p.k_hi = float(k);
  if (double(p.k_hi) > k) p.k_hi = std::nextafterf(p.k_hi, 0.f);
  // (above zero, so that -infinity stays -infinity under both; by no more than the smallest number, as logits may be large where the scale is small)
  p.k_lo = std::max(float(k - double(p.k_hi)), std::numeric_limits<float>::denorm_min());
  // Rows are cut into equal parts so that the teams' rounds are even and short; a round costs its tiles and about BS_ITEM_COST more for the item's end.
  const int64_t rows = int64_t(a.n_requests) * a.n_beams;
  const int per = a.type == HS_TYPE_F32 ? 4 : 8, tiles = (a.vocab + per - 1 + BS_TILE_PIECES * per - 1) / (BS_TILE_PIECES * per);
  const int64_t teams = int64_t(share_count(sm_count)) * BS_TEAMS;
  int64_t least = -1;
  p.parts = 1;
  for (int parts = 1; parts <= std::min(tiles, BS_MAX_PARTS) && rows * parts <= std::max(rows, 4 * teams); ++parts) {
    const int64_t cost = (rows * parts + teams - 1) / teams * ((tiles + parts - 1) / parts + BS_ITEM_COST);
    if (least < 0 || cost < least) {
      least = cost;
      p.parts = parts;
    }
  }
  p.items = int(rows * p.parts);
  for (p.lanes = 1; p.lanes < std::min(p.parts, 32); p.lanes *= 2) {}
  const int grid = int(std::min<int64_t>(sm_budget, p.items));
  return launch_step_kernel(pick(a.type), grid, BS_THREADS, kSelectSmem, stream, true, p);
}

}  // namespace hs
