// Attention of one new token per sequence over the paged cache, planned on the device.
//
//   group     (sequence, KV head, up to 8 NT of its query heads): the pages that its rows see, in key order.  Groups follow one another
//             sequence by sequence; all their pages together are one line of work.
//   share     what a block does at a time: whole groups, a part of one group, or an equal piece of the line that is cut anywhere, by a rule on the lengths (below);
//             about one per SM of the device.  A share is cut into eight equal pieces, one per warp: every warp of it has the same number of
//             pages, give or take one.  Where the cuts lie depends on the lengths and the device, never on the budget, and a block takes one share
//             after the other.
//   warp      streams its pages through a ring of its own in shared memory (one bulk tensor copy brings the K and the V block of a
//             page and head), lane 0 issuing ahead; mma.sync tiles with keys as rows and heads as columns, softmax in the log2 domain with
//             a running maximum and sum per head.  A group that lies within a warp's piece is finished there.
//   joins     a group that is cut leaves one partial result (output, maximum, sum per head) per warp; the block adds those of a
//             share in order, and the block that delivers the last share of a group the shares', in order.
//
// It is the cache's bytes that bound it where there are many -- 64 sequences of 512 .. 4096 keys, 28 heads on 4 of 128: 312 MB in 63 us, 4.9 TB/s, three quarters of what a
// copy reaches --, and latency where there are few: 6.7 us for two short sequences, of which the launch is half and the rest one round trip
// each for lengths, page ids and pages, and a join.
//
// Every block plans for itself: page counts of all sequences, one running sum in shared memory, and 32 pages at a time are looked
// up by a warp's lanes, each finding the sequence of its page by bisection.
#include <math.h>

#include <algorithm>

#include "paged_scores.cuh"

namespace hs {
namespace {

constexpr int PD_WARPS = 8, PD_THREADS = PD_WARPS * 32;
constexpr int PD_RING_BYTES = 192 * 1024;
constexpr int PD_MIN_PAGES = 16;                 // of a share: two per warp
// How the line is cut, by what the longest share has to do in pages: a join of shares takes as long as PD_JOIN_COST pages and one for each part; cuts inside
// groups, which give a block two groups and two joins, as PD_CUT_COST.  us by groups / anywhere: 2 sequences of 81 keys, 16 heads on 4 of 128, 6.7 /
// 13.4; 16 of 128 .. 1024, 16 on 4 of 64, 12.0 / 14.3; 3 of 20001 .. 32768, 16 on 2 of 128, 23.8 / 29.0; 64 of 512 .. 4096, 28 on 4 of 128, 68.0 / 63.1;
// 47 of 2713, 28 on 4 of 64, 47.6 / 38.6.
constexpr int PD_MIN_PART = 8, PD_JOIN_COST = 20, PD_CUT_COST = 66;
constexpr int PD_WORDS = 160;                     // 32-bit words of shared memory in front of the sequences' page counts
constexpr float kLn2 = 0.6931471805599453f;

struct DecodeParams {
  CUtensorMap tm;
  hs_paged_attention_t a;
  ScoreScale score;
  int shares, chunks;                            // chunks: groups per KV head
  int groups, parts;                             // most whole groups that a share can have; parts of a group that there are shares for
};

template <int DH>
struct PageGeom {
  static constexpr int HALVES = DH / 64;
  static constexpr int BYTES = HALVES * 2048;    // K (or V): [half][16 keys][128 bytes], 128-byte swizzle
  static constexpr int SLOT = 2 * BYTES;
  static constexpr int SLOTS = PD_RING_BYTES / PD_WARPS / SLOT;
};
__device__ __forceinline__ int page_off(int key, int chunk) {       // of a 16-byte chunk of a key's row
  return (chunk >> 3) * 2048 + key * 128 + (((chunk & 7) ^ (key & 7)) << 4);
}
// The K and the V block of a page and head: read once in a step, so they are the first to leave the L2 again (the kernel's own code and the
// partial results stay).
__device__ __forceinline__ void load_page(void* dst, const CUtensorMap* m, uint64_t* bar, int row, int layer) {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %3, %5}], [%2], %6;"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(0), "r"(row), "r"(layer * 2), "l"(policy)
      : "memory");
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t t;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
  return t;
}
__device__ __forceinline__ float columns_max(float v) {             // over the eight lanes that share lane % 4
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
}
__device__ __forceinline__ float columns_sum(float v) {
  v += __shfl_xor_sync(0xffffffffu, v, 4);
  v += __shfl_xor_sync(0xffffffffu, v, 8);
  return v + __shfl_xor_sync(0xffffffffu, v, 16);
}
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// One partial result: ROWS heads of DH outputs relative to the maximum, then (maximum in log2 units, sum) per head.
template <int DH, int ROWS>
struct PartOf {
  float o[ROWS][DH + 4];                                 // (four floats more: the warps write and read these without bank conflicts where they are in shared memory)
  float2 ml[ROWS];
};
// Reads of partial results, in shared memory or in global memory where another SM has written them.
__device__ __forceinline__ float4 load_part(const float* p) {
  float4 v;
  asm volatile("ld.relaxed.gpu.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float2 load_part(const float2* p) {
  float2 v;
  asm volatile("ld.relaxed.gpu.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p) : "memory");
  return v;
}

// A group's running softmax in a warp.  This lane holds heads 8 t + 2 (lane % 4) and the next one, of the scores keys lane / 4 and lane / 4 + 8, of the
// outputs coordinates lane / 4 and lane / 4 + 8 of every sixteen.
template <int DH, int NT, bool F16, bool MOD>
struct GroupState {
  uint32_t qf[DH / 16][NT][2];
  float o[DH / 16][NT][4], m[NT][2], l[NT][2];
  float slope[NT][2];

  __device__ __forceinline__ void begin(const uint16_t* q, const float* slopes, int heads, int lane) {
    const int hq = lane >> 2;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int ks = 0; ks < DH / 16; ++ks)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          qf[ks][t][e] = 8 * t + hq < heads ? *reinterpret_cast<const uint32_t*>(q + (8 * t + hq) * DH + ks * 16 + 8 * e + 2 * (lane & 3)) : 0u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[t][e] = -INFINITY;
        l[t][e] = 0.f;
        const int h = 8 * t + 2 * (lane & 3) + e;
        if (MOD) slope[t][e] = slopes && h < heads ? slopes[h] * 1.4426950408889634f : 0.f;
      }
#pragma unroll
      for (int j = 0; j < DH / 16; ++j) o[j][t][0] = o[j][t][1] = o[j][t][2] = o[j][t][3] = 0.f;
    }
  }

  // One page in shared memory.  seen: bit k = key k is seen; dist: p - (the page's first key).
  __device__ __forceinline__ void page(uint32_t k_base, uint32_t v_base, uint32_t seen, int dist, const ScoreScale& sc, int lane) {
    const int key = lane >> 2;
    float s[NT][4], s2[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = s2[t][e] = 0.f;
    {
      const int kk = (lane & 7) + ((lane >> 3) & 1) * 8, cc = lane >> 4;
#pragma unroll
      for (int ks = 0; ks < DH / 16; ks += 2) {
        uint32_t kf[4], kg[4];
        ldmatrix_x4(kf, k_base + page_off(kk, 2 * ks + cc));
        ldmatrix_x4(kg, k_base + page_off(kk, 2 * ks + 2 + cc));
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma_16816<F16>(s[t], kf, qf[ks][t][0], qf[ks][t][1]);
          mma_16816<F16>(s2[t], kg, qf[ks + 1][t][0], qf[ks + 1][t][1]);
        }
      }
    }
    uint32_t vf[DH / 16][4];
    {
      const int kk = (lane & 7) + (lane >> 4) * 8, cc = (lane >> 3) & 1;
#pragma unroll
      for (int dp = 0; dp < DH / 16; ++dp) ldmatrix_x4_trans(vf[dp], v_base + page_off(kk, 2 * dp + cc));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = (s[t][e] + s2[t][e]) * sc.in;
        if (MOD) {
          if (sc.out != 0.f) x = sc.out * tanh_any(x);
          x = fmaf(-slope[t][e & 1], fabsf(float(dist - key - 8 * (e >> 1))), x);
        }
        s[t][e] = x;
      }
    if (seen != 0xffffu) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!((seen >> (key + 8 * (e >> 1))) & 1u)) s[t][e] = -INFINITY;
      // what the cache holds at keys that are not seen may be anything: it must not meet the weight 0
#pragma unroll
      for (int dp = 0; dp < DH / 16; ++dp)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t two = seen >> (2 * (lane & 3) + 8 * (e >> 1));
          vf[dp][e] &= ((two & 1u) ? 0x0000ffffu : 0u) | ((two & 2u) ? 0xffff0000u : 0u);
        }
    }
    bool up = false;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) up |= fmaxf(s[t][e], s[t][e + 2]) > m[t][e];
    if (__any_sync(0xffffffffu, up)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float mn = fmaxf(m[t][e], columns_max(fmaxf(s[t][e], s[t][e + 2])));
          const float al = fast_exp2(m[t][e] - finite_or_zero(mn));
          m[t][e] = mn;
          l[t][e] *= al;
#pragma unroll
          for (int j = 0; j < DH / 16; ++j) {
            o[j][t][e] *= al;
            o[j][t][e + 2] *= al;
          }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = fast_exp2(s[t][e] - finite_or_zero(m[t][e & 1]));
        l[t][e & 1] += s[t][e];
      }
      // (the weights are at most 1 here and get 8 or 11 bits, which the product with v in 16 bits takes; their sum, above, keeps fp32.  o is off by 2^-8 of the
      // largest |v| (2^-11) at most, usually far less: 0.0017 of the outputs' spread against 64 bits in bf16, which rounding o alone leaves too)
      const uint32_t p0 = transpose_8x8(pack_16<F16>(s[t][0], s[t][1])), p1 = transpose_8x8(pack_16<F16>(s[t][2], s[t][3]));
#pragma unroll
      for (int dp = 0; dp < DH / 16; ++dp) mma_16816<F16>(o[dp][t], vf[dp], p0, p1);
    }
  }

  // The group's part of this warp.
  __device__ __forceinline__ void put(PartOf<DH, 8 * NT>* part, int heads, int lane) {
    const int d = lane >> 2;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int h = 8 * t + 2 * (lane & 3) + e;
        const float sum = columns_sum(l[t][e]);
        if (h >= heads) continue;
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) {
          part->o[h][16 * j + d] = o[j][t][e];
          part->o[h][16 * j + d + 8] = o[j][t][e + 2];
        }
        if (d == 0) part->ml[h] = make_float2(m[t][e], sum);
      }
  }
  // The finished rows of a group that was not cut.
  __device__ __forceinline__ void store(uint16_t* out, float* lse, int heads, int lane) {
    const int d = lane >> 2;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int h = 8 * t + 2 * (lane & 3) + e;
        const float sum = columns_sum(l[t][e]);
        if (h >= heads) continue;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) {
          const uint32_t w = pack_16<F16>(o[j][t][e] * inv, o[j][t][e + 2] * inv);
          out[h * DH + 16 * j + d] = uint16_t(w);
          out[h * DH + 16 * j + d + 8] = uint16_t(w >> 16);
        }
        if (d == 0 && lse) lse[h] = sum == 0.f ? -INFINITY : kLn2 * (m[t][e] + log2f(sum));
      }
  }
};

// What a warp's piece of the line leaves to be joined: the part of a group that began in front of the piece (place 0), and of one that
// goes on behind it (place 1).
struct Cut {
  int g0, g1;                                            // the group's place in the line; g1 = 0: nothing
  void* part;
  int row, head0, heads, group;                          // group: its number, sequence by sequence
};

template <int DH, int NT, bool F16, bool MOD>
__global__ void __launch_bounds__(PD_THREADS, 1) paged_decode_kernel(const __grid_constant__ DecodeParams p) {
  using G = PageGeom<DH>;
  using Part = PartOf<DH, 8 * NT>;
  constexpr int SLOTS = G::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_all = reinterpret_cast<uint64_t*>(smem + PD_RING_BYTES);
  int* words = reinterpret_cast<int*>(full_all + PD_WARPS * SLOTS);
  volatile int* abort_flag = words;
  int* last = words + 1;                                 // of the runs, those whose shares this block joins
  int *warp_sum = words + 2, *warp_max = words + 10;     // [8] each
  Cut(*cuts)[2] = reinterpret_cast<Cut(*)[2]>(words + 20);              // [8][2]
  int* page_begin = words + PD_WORDS;                    // [n_seqs + 1]
  const hs_paged_attention_t& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n = a.n_seqs, heads_all = a.n_q_heads / a.n_kv_heads, units = a.n_kv_heads * p.chunks;

  if (tid == 0) {
    for (int i = 0; i < PD_WARPS * SLOTS; ++i) mbar_init(&full_all[i], 1);
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&p.tm);
  }
  griddep_wait();

  // ---------------------------------------------------------------- the plan
  int most_pages = 0;                                    // of a group
  {
    const int per = (n + PD_THREADS - 1) / PD_THREADS, s0 = tid * per;
    int mine = 0, longest = 0;
    for (int i = 0; i < per; ++i) {
      const int s = s0 + i;
      if (s >= n) break;
      const SeqView v = view_seq(a, s);
      if (v.error && blockIdx.x == 0) atomicExch(a.status, v.error);
      const int pages = v.rows > 0 ? page_runs(v, v.kv - 1, v.kv - 1, a.window).total() : 0;
      if (v.rows > 0 && pages == 0 && s % gridDim.x == blockIdx.x) {       // a row that sees nothing
        for (int h = 0; h < a.n_q_heads; ++h) {
          uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.o) + v.row * a.o_stride + h * DH);
          for (int c = 0; c < DH / 8; ++c) o[c] = make_uint4(0, 0, 0, 0);
          if (a.lse) a.lse[int64_t(v.row) * a.n_q_heads + h] = -INFINITY;
        }
      }
      page_begin[s] = mine;
      mine += pages;
      longest = max(longest, pages);
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == 31) {
      warp_sum[warp] = inc;
      warp_max[warp] = longest;
    }
    __syncthreads();
    int before = inc - mine, total = 0;
    for (int w = 0; w < PD_WARPS; ++w) {
      if (w < warp) before += warp_sum[w];
      total += warp_sum[w];
      most_pages = max(most_pages, warp_max[w]);
    }
    for (int i = 0; i < per && s0 + i < n; ++i) page_begin[s0 + i] += before;
    if (tid == 0) page_begin[n] = total;
    __syncthreads();
  }
  // (the host has seen to it that places in the line are 32-bit numbers.)  Shares are whole groups, p.groups or one fewer each; or parts of `part` pages
  // of a group, as many shares for each as the longest has parts; or equal pieces of the line, the first `more` ones with one page more.
  const int line = page_begin[n] * units, equal = max(line / p.shares, PD_MIN_PAGES);
  const int parts = min(p.parts, max(int(sqrtf(float(most_pages))), 1)), part = max((most_pages + parts - 1) / parts, PD_MIN_PART);
  const int whole_cost = p.groups * most_pages, part_cost = p.parts > 1 ? part + PD_JOIN_COST + parts : whole_cost;
  const bool by_groups = min(whole_cost, part_cost) <= equal + PD_JOIN_COST + PD_CUT_COST + most_pages / equal;
  const int per_group = !by_groups ? 0 : whole_cost <= part_cost ? 1 : (most_pages + part - 1) / part;        // shares; 1: whole groups
  const int cuttable = per_group == 0 ? line : n * units * per_group;
  const int shares = per_group == 0 ? min(p.shares, max(1, line / PD_MIN_PAGES)) : min(p.shares, cuttable), base = cuttable / shares, more = cuttable - base * shares;
  auto group_begin = [&](int g) {
    const int s = min(g / units, n), pages = s < n ? page_begin[s + 1] - page_begin[s] : 0;
    return page_begin[s] * units + (g - s * units) * pages;
  };
  auto share_begin = [&](int b) {
    if (per_group > 1) {
      const int g = b / per_group, s = min(g / units, n), pages = s < n ? page_begin[s + 1] - page_begin[s] : 0;
      return page_begin[s] * units + (g - s * units) * pages + min((b - g * per_group) * part, pages);
    }
    const int x = base * b + min(b, more);
    return per_group == 1 ? group_begin(x) : x;
  };
  auto share_of = [&](int x) { return x < more * (base + 1) ? x / (base + 1) : more + (x - more * (base + 1)) / max(base, 1); };
  auto first_share = [&](int g0, int group) { return per_group > 1 ? group * per_group : share_of(g0); };          // of a divided group
  auto last_share = [&](int g0, int g1, int group) { return per_group > 1 ? group * per_group + (g1 - g0 - 1) / part : share_of(g1 - 1); };

  Part* warp_parts = reinterpret_cast<Part*>(static_cast<char*>(a.workspace) + kWsScratch);          // [share][warp]
  Part* share_parts = warp_parts + size_t(kMaxShares) * PD_WARPS;                                    // [share][2]
  int* done_words = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsAttnDone);

  uint8_t* ring = smem + warp * SLOTS * G::SLOT;
  uint64_t* full = full_all + warp * SLOTS;
  int fill = 0, cur = 0;
  uint32_t phase = 0;
  bool ok = true;

  // A page of the line, as one lane knows it.
  struct Item {
    int coord;           // first row of the page's K block for the head in the tensor map, or -1: a page id outside the pool
    int group_seq, group_unit;
    int key0;
  };
  auto find_seq = [&](int x) {                           // the sequence of a place in the line
    const int y = x / units;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (page_begin[mid] <= y) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  auto look_up = [&](int x, int end) {
    Item it = {-1, 0, 0, 0};
    if (unsigned(x) < unsigned(end)) {                   // (x may be up to 64 places behind a line that ends just below 2^31)
      const int s = find_seq(x), pages = page_begin[s + 1] - page_begin[s];
      const int r = x - page_begin[s] * units;
      const int unit = r / pages, i = r - unit * pages;
      const SeqView v = view_seq(a, s);
      const int logical = page_runs(v, v.kv - 1, v.kv - 1, a.window).page(i);
      const int id = a.block_tables[int64_t(s) * a.max_pages_per_seq + logical];
      it.group_seq = s;
      it.group_unit = unit;
      it.key0 = logical * 16;
      if (id >= 0 && id < a.num_pages) it.coord = (id * a.n_kv_heads + unit / p.chunks) * 16;
      else atomicExch(a.status, kErrBadBlockTable);
    }
    return it;
  };
  auto request = [&](int coord) {                        // lane 0
    mbar_expect_tx(&full[fill], G::SLOT);
    load_page(ring + fill * G::SLOT, &p.tm, &full[fill], max(coord, 0), a.layer);
    if (++fill == SLOTS) fill = 0;
  };

  for (int share = blockIdx.x; share < shares; share += gridDim.x) {
    const int b0 = share_begin(share), b1 = share_begin(share + 1);
    const int piece = (b1 - b0) / PD_WARPS, longer = (b1 - b0) % PD_WARPS;       // (the first `longer` warps have one page more)
    auto piece_begin = [&](int w) { return b0 + piece * w + min(w, longer); };
    const int w0 = piece_begin(warp), w1 = piece_begin(warp + 1);
    Item now = look_up(w0 + lane, w1);
    const int n_pages = w1 - w0;
    if (lane < 2) cuts[warp][lane].g1 = 0;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) {
      const int c = __shfl_sync(0xffffffffu, now.coord, i);
      if (lane == 0 && i < n_pages) request(c);
    }
    Item next = look_up(w0 + 32 + lane, w1);
    GroupState<DH, NT, F16, MOD> st;
    int seq = -1, unit = -1, heads = 0, from = 0, pos = 0, prefix = 0;
    const uint16_t* q = nullptr;
    int64_t row = 0;
    int g0 = 0, g1 = 0;                                  // the group's place in the line
    auto finish = [&](bool at_end) {                     // the group that the warp has come to the end of, or of its part of
      if (g0 >= w0 && g1 <= w1) {
        const int head0 = (unit / p.chunks) * heads_all + (unit % p.chunks) * 8 * NT;
        st.store(static_cast<uint16_t*>(a.o) + row * a.o_stride + head0 * DH, a.lse ? a.lse + row * a.n_q_heads + head0 : nullptr, heads, lane);
      } else {
        const int slot = g0 >= w0 ? 1 : 0;
        // (at the end of its piece the warp's ring is idle and takes the part; before that it goes to the workspace)
        Part* part = at_end ? reinterpret_cast<Part*>(ring) : warp_parts + share * PD_WARPS + warp;
        st.put(part, heads, lane);
        if (lane == 0) cuts[warp][slot] = Cut{g0, g1, part, int(row), (unit / p.chunks) * heads_all + (unit % p.chunks) * 8 * NT, heads, seq * units + unit};
      }
    };
    for (int i = 0; i < n_pages; ++i) {
      const int j = i & 31;
      if (j == 0 && i > 0) {
        now = next;
        next = look_up(w0 + i + 32 + lane, w1);
      }
      {
        const int k = j + SLOTS - 1;
        const int c0 = __shfl_sync(0xffffffffu, now.coord, k & 31), c1 = __shfl_sync(0xffffffffu, next.coord, k & 31);
        if (lane == 0 && i + SLOTS - 1 < n_pages) request(k < 32 ? c0 : c1);
      }
      const int s = __shfl_sync(0xffffffffu, now.group_seq, j), g = __shfl_sync(0xffffffffu, now.group_unit, j);
      const int key0 = __shfl_sync(0xffffffffu, now.key0, j), coord = __shfl_sync(0xffffffffu, now.coord, j);
      if (s != seq || g != unit) {
        if (seq >= 0) finish(false);
        seq = s;
        unit = g;
        const SeqView v = view_seq(a, s);
        pos = v.kv - 1;
        from = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
        prefix = v.prefix;
        row = v.row;
        const int pages = page_begin[s + 1] - page_begin[s];
        g0 = page_begin[s] * units + unit * pages;
        g1 = g0 + pages;
        const int in_head = (unit % p.chunks) * 8 * NT, head0 = (unit / p.chunks) * heads_all + in_head;
        heads = min(heads_all - in_head, 8 * NT);
        q = static_cast<const uint16_t*>(a.q) + row * a.q_stride + head0 * DH;
        st.begin(q, a.slopes ? a.slopes + head0 : nullptr, heads, lane);
      }
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&full[cur], phase, abort_flag, a.status));
      const uint32_t k_base = smem_u32(ring + cur * G::SLOT);
      if (++cur == SLOTS) { cur = 0; phase ^= 1; }
      uint32_t seen = 0xffffu;
      if (key0 + 15 > pos) seen = (1u << (pos + 1 - key0)) - 1u;
      if (key0 < from) {
        uint32_t hidden = from - key0 >= 16 ? 0xffffu : (1u << (from - key0)) - 1u;
        if (key0 < prefix) hidden &= prefix - key0 >= 16 ? 0u : ~((1u << (prefix - key0)) - 1u);
        seen &= ~hidden;
      }
      if (coord < 0) seen = 0;
      if (ok) st.page(k_base, k_base + G::BYTES, seen, pos - key0, p.score, lane);
      __syncwarp();                                      // every lane is done with the slot before lane 0 asks for its next page
    }
    if (seq >= 0) finish(true);
    __threadfence_block();
    __syncthreads();
    // --------------------------------------------------------------- the joins
    // A run of parts begins with a warp whose group goes on behind its piece (place 1), or, at the share's beginning, with the group that was
    // cut there (place 0); the next warps' parts of it are in their places 0.  First the parts of this share are joined, then, where this block is the
    // last one of a group's to come, the shares' -- by the same instructions: this code runs once a launch, and what it took was the time to fetch it.
    const int my_g0 = lane < 2 * PD_WARPS ? cuts[lane >> 1][lane & 1].g0 : 0, my_g1 = lane < 2 * PD_WARPS ? cuts[lane >> 1][lane & 1].g1 : 0;
    const int my_group = lane < 2 * PD_WARPS ? cuts[lane >> 1][lane & 1].group : 0;
    const bool begins = my_g1 > 0 && (lane == 0 || (lane & 1));          // (of each warp's lanes: a place that a run begins with)
    unsigned todo = __ballot_sync(0xffffffffu, begins);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      if (pass == 1) {
        // the groups that other shares have parts of: the one cut at the share's beginning, the one cut at its end
        todo = __ballot_sync(0xffffffffu, begins && (my_g0 < b0 || my_g1 > b1));
        if (todo == 0) break;
        __threadfence();
        __syncthreads();
        bool is_last = false;
        if (warp == 0 && todo >> lane & 1u) {
          const int f = first_share(my_g0, my_group), e = last_share(my_g0, my_g1, my_group);
          is_last = atomicAdd(done_words + f, 1) == e - f;
          if (is_last) done_words[f] = 0;                // ready for the next call
        }
        if (warp == 0) {
          const unsigned mine = __ballot_sync(0xffffffffu, is_last);
          if (lane == 0) *last = int(mine);
        }
        __syncthreads();
        todo = unsigned(*last);
        if (todo == 0) break;
        __threadfence();
      }
#pragma unroll 1
      for (; todo; todo &= todo - 1) {
        const int k = __ffs(todo) - 1, w = k >> 1, slot = k & 1;
        const int g0 = __shfl_sync(0xffffffffu, my_g0, k), g1 = __shfl_sync(0xffffffffu, my_g1, k);
        const Cut& cut = cuts[w][slot];
        const bool within = g0 >= b0 && g1 <= b1;
        int n_parts = 1, f = 0;
        if (pass == 0) {
          n_parts += __popc(__ballot_sync(0xffffffffu, !(lane & 1) && lane > k && my_g1 > 0 && my_g0 == g0));
        } else {
          f = first_share(g0, cut.group);
          n_parts = last_share(g0, g1, cut.group) - f + 1;
        }
#pragma unroll 1
        for (int i = tid; i < cut.heads * (DH / 4); i += PD_THREADS) {
          const int h = i / (DH / 4), c = i % (DH / 4) * 4;
          float m = -INFINITY, l = 0.f;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int j0 = 0; j0 < n_parts; j0 += 8) {      // eight parts on their way at a time
            float2 ml[8];
            float4 ov[8];
            float mn = m;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int j = min(j0 + u, n_parts - 1);
              const Part* part = pass == 1 ? share_parts + (f + j) * 2 + (j == 0 ? 1 : 0) : static_cast<const Part*>(cuts[w + j][j == 0 ? slot : 0].part);
              ml[u] = load_part(&part->ml[h]);
              ov[u] = load_part(&part->o[h][c]);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              if (j0 + u >= n_parts) ml[u] = make_float2(-INFINITY, 0.f);
              mn = fmaxf(mn, ml[u].x);
            }
            const float zero = finite_or_zero(mn), f0 = fast_exp2(m - zero);
            m = mn;
            l *= f0; o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float f = fast_exp2(ml[u].x - zero);         // (0 for a part that is not there; its outputs are another part's)
              l = fmaf(f, ml[u].y, l);
              o.x = fmaf(f, ov[u].x, o.x);
              o.y = fmaf(f, ov[u].y, o.y);
              o.z = fmaf(f, ov[u].z, o.z);
              o.w = fmaf(f, ov[u].w, o.w);
            }
          }
          if (within || pass == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o) + int64_t(cut.row) * a.o_stride + (cut.head0 + h) * DH + c) =
                make_uint2(pack_16<F16>(o.x * inv, o.y * inv), pack_16<F16>(o.z * inv, o.w * inv));
            if (c == 0 && a.lse) a.lse[int64_t(cut.row) * a.n_q_heads + cut.head0 + h] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
          } else {
            Part* mine = share_parts + share * 2 + slot;
            __stcg(reinterpret_cast<float4*>(&mine->o[h][c]), o);
            if (c == 0) __stcg(&mine->ml[h], make_float2(m, l));
          }
        }
      }
    }
    fence_proxy_async();
    __syncthreads();
  }
  if (*abort_flag) drain_after_abort();
}

template <int DH>
constexpr int pd_smem() {
  return 1024 + PD_RING_BYTES + PD_WARPS * PageGeom<DH>::SLOTS * 8 + PD_WORDS * 4 + (HS_DEVICE_MAX_SEQS + 1) * 4;
}
static_assert(pd_smem<64>() <= 227 * 1024 && pd_smem<128>() <= 227 * 1024, "fits one SM");
static_assert(size_t(kMaxShares) * (PD_WARPS + 2) * sizeof(PartOf<128, 16>) <= kWsScratchBytes, "parts of warps and shares");
static_assert(kWsAttnDone + kMaxShares * 4 <= kWsLogprobsDone, "one word per share");

using DecodeKernel = void (*)(DecodeParams);
template <int DH, int NT>
DecodeKernel pick(bool f16, bool mod) {
  if (f16) return mod ? paged_decode_kernel<DH, NT, true, true> : paged_decode_kernel<DH, NT, true, false>;
  return mod ? paged_decode_kernel<DH, NT, false, true> : paged_decode_kernel<DH, NT, false, false>;
}
DecodeKernel pick(int dh, bool two, bool f16, bool mod) {
  if (dh == 128) return two ? pick<128, 2>(f16, mod) : pick<128, 1>(f16, mod);
  return two ? pick<64, 2>(f16, mod) : pick<64, 1>(f16, mod);
}

}  // namespace

cudaError_t paged_decode_set_attributes() {
  for (int i = 0; i < 16; ++i) {
    const int dh = i & 1 ? 128 : 64;
    const cudaError_t e = set_kernel_smem(pick(dh, i & 2, i & 4, i & 8), dh == 128 ? pd_smem<128>() : pd_smem<64>());
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_paged_decode(const hs_paged_attention_t& a, const CUtensorMap& tm_kv_page, int sm_count, int sm_budget, cudaStream_t stream) {
  DecodeParams p{};
  p.tm = tm_kv_page;
  p.a = a;
  p.score = score_scale(a.scale, a.cap);
  p.shares = share_count(sm_count);
  const int heads = a.n_q_heads / a.n_kv_heads;
  const bool two = heads > 8;
  p.chunks = (heads + (two ? 16 : 8) - 1) / (two ? 16 : 8);
  const int n_groups = a.n_seqs * a.n_kv_heads * p.chunks;
  p.groups = (n_groups + p.shares - 1) / p.shares;
  p.parts = std::max(p.shares / n_groups, 1);
  const int grid = std::min(p.shares, sm_budget);
  return launch_step_kernel(pick(a.head_dim, two, a.type == HS_TYPE_F16, a.cap > 0.f || a.slopes != nullptr), grid, PD_THREADS,
                            a.head_dim == 128 ? pd_smem<128>() : pd_smem<64>(), stream, true, p);
}

}  // namespace hs
