// Attention of one new token per sequence over the paged cache, planned on the device.
//
//   group     (sequence, KV head, up to 8 NT of its query heads): the pages that its rows see, in key order.  Groups follow one another
//             sequence by sequence; all their pages together are one line of work.
//   share     the line is cut into one equal piece per SM of the device, a share into eight equal pieces, one per warp: every
//             warp has the same number of pages, give or take one, whatever the lengths.  Where the cuts lie depends on the
//             lengths and the device, never on the budget, and a block takes one share after the other.
//   warp      streams its pages through a ring of its own in shared memory (one bulk tensor copy brings the K and the V block of a
//             page and head), lane 0 issuing ahead; mma.sync tiles with keys as rows and heads as columns, softmax in the log2 domain with
//             a running maximum and sum per head.  A group that lies within a warp's piece is finished there.
//   joins     a group that is cut leaves one partial result (output, maximum, sum per head) per warp; the block adds those of a
//             share in order, and the block that delivers the last share of a group the shares', in order.
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
constexpr float kLn2 = 0.6931471805599453f;

struct DecodeParams {
  CUtensorMap tm;
  hs_paged_attention_t a;
  ScoreScale score;
  int shares, chunks;                            // chunks: groups per KV head
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
  float o[ROWS][DH];
  float2 ml[ROWS];
};

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

// Adds parts first, first + 1, .. in order, two columns a thread; every thread of the block.  emit(head, column, o0, o1, max, sum).
template <int DH, int ROWS, typename At, typename Emit>
__device__ __forceinline__ void join_parts(int n, int heads, At at, Emit emit) {
  for (int i = threadIdx.x; i < heads * (DH / 2); i += PD_THREADS) {
    const int h = i / (DH / 2), c = 2 * (i - h * (DH / 2));
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j0 = 0; j0 < n; j0 += 8) {                  // eight on their way at a time
      float2 ml[8], ov[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const PartOf<DH, ROWS>* part = at(min(j0 + u, n - 1));
        ml[u] = __ldcg(&part->ml[h]);
        ov[u] = __ldcg(reinterpret_cast<const float2*>(&part->o[h][c]));
      }
      float mn = m;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (j0 + u < n) mn = fmaxf(mn, ml[u].x);
      const float f0 = fast_exp2(m - finite_or_zero(mn));
      m = mn;
      l *= f0; o0 *= f0; o1 *= f0;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (j0 + u < n) {
          const float f = fast_exp2(ml[u].x - finite_or_zero(m));
          l = fmaf(f, ml[u].y, l);
          o0 = fmaf(f, ov[u].x, o0);
          o1 = fmaf(f, ov[u].y, o1);
        }
    }
    emit(h, c, o0, o1, m, l);
  }
}

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
  int* flag = words + 1;
  int* warp_sum = words + 2;                             // [8]
  int* cut = words + 16;                                 // [9][3]: runs of partial results of the share
  int* page_begin = words + 64;                          // [n_seqs + 1]
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
  {
    const int per = (n + PD_THREADS - 1) / PD_THREADS, s0 = tid * per;
    int mine = 0;
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
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    int before = inc - mine, total = 0;
    for (int w = 0; w < PD_WARPS; ++w) {
      if (w < warp) before += warp_sum[w];
      total += warp_sum[w];
    }
    for (int i = 0; i < per && s0 + i < n; ++i) page_begin[s0 + i] += before;
    if (tid == 0) page_begin[n] = total;
    __syncthreads();
  }
  const int64_t line = int64_t(page_begin[n]) * units;
  const int shares = int(min(int64_t(p.shares), max(int64_t(1), line / PD_MIN_PAGES)));
  auto share_begin = [&](int b) { return line * b / shares; };
  auto share_of = [&](int64_t x) { return int(((x + 1) * shares - 1) / line); };

  Part* warp_parts = reinterpret_cast<Part*>(static_cast<char*>(a.workspace) + kWsScratch);          // [share][warp][2]
  Part* share_parts = warp_parts + size_t(kMaxShares) * PD_WARPS * 2;                                // [share][2]
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
  auto find_seq = [&](int64_t x) {                       // the sequence of a place in the line
    const int y = int(x / units);
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (page_begin[mid] <= y) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  auto look_up = [&](int64_t x, int64_t end) {
    Item it = {-1, 0, 0, 0};
    if (x < end) {
      const int s = find_seq(x), pages = page_begin[s + 1] - page_begin[s];
      const int r = int(x - int64_t(page_begin[s]) * units);
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
    tma_load_4d(ring + fill * G::SLOT, &p.tm, &full[fill], 0, max(coord, 0), 0, a.layer * 2);
    if (++fill == SLOTS) fill = 0;
  };

  for (int share = blockIdx.x; share < shares; share += gridDim.x) {
    const int64_t b0 = share_begin(share), b1 = share_begin(share + 1);
    const int64_t w0 = b0 + (b1 - b0) * warp / PD_WARPS, w1 = b0 + (b1 - b0) * (warp + 1) / PD_WARPS;
    Item now = look_up(w0 + lane, w1), next = look_up(w0 + 32 + lane, w1);
    const int n_pages = int(w1 - w0);
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) {
      const int c = __shfl_sync(0xffffffffu, now.coord, i);
      if (lane == 0 && i < n_pages) request(c);
    }
    GroupState<DH, NT, F16, MOD> st;
    int seq = -1, unit = -1, heads = 0, from = 0, pos = 0, prefix = 0;
    const uint16_t* q = nullptr;
    int64_t row = 0;
    int64_t g0 = 0, g1 = 0;                              // the group's place in the line
    auto finish = [&]() {                                // the group that the warp has come to the end of, or of its part of
      if (g0 >= w0 && g1 <= w1) {
        const int head0 = (unit / p.chunks) * heads_all + (unit % p.chunks) * 8 * NT;
        st.store(static_cast<uint16_t*>(a.o) + row * a.o_stride + head0 * DH, a.lse ? a.lse + row * a.n_q_heads + head0 : nullptr, heads, lane);
      } else {
        st.put(warp_parts + (share * PD_WARPS + warp) * 2 + (g0 >= w0 ? 1 : 0), heads, lane);
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
        if (seq >= 0) finish();
        seq = s;
        unit = g;
        const SeqView v = view_seq(a, s);
        pos = v.kv - 1;
        from = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
        prefix = v.prefix;
        row = v.row;
        const int pages = page_begin[s + 1] - page_begin[s];
        g0 = int64_t(page_begin[s]) * units + int64_t(unit) * pages;
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
    if (seq >= 0) finish();
    __threadfence_block();
    __syncthreads();
    // --------------------------------------------------------------- the joins
    // Runs of parts in this share: part (warp, end), then (warp + 1, 0), .. of one group.  Every thread walks the eight warps' cuts.
    int w = 0;
    while (w < PD_WARPS) {
      const int64_t c0 = b0 + (b1 - b0) * w / PD_WARPS, c1 = b0 + (b1 - b0) * (w + 1) / PD_WARPS;
      if (c0 == c1) { ++w; continue; }
      // the group at the end of warp w's piece (a part of it that begins here), or, for the first warp, the one cut in front of it
      auto group_at = [&](int64_t x, int64_t& lo, int64_t& hi, int& s, int& g) {
        s = find_seq(x);
        const int pages = page_begin[s + 1] - page_begin[s];
        const int64_t base = int64_t(page_begin[s]) * units;
        g = int((x - base) / pages);
        lo = base + int64_t(g) * pages;
        hi = lo + pages;
      };
      auto join_run = [&](int first_warp, int first_end, int64_t lo, int64_t hi, int s, int g) {
        int last_warp = first_warp;
        while (last_warp + 1 < PD_WARPS && b0 + (b1 - b0) * (last_warp + 1) / PD_WARPS < hi) ++last_warp;
        // (pieces of no page between them deliver nothing)
        int count = 0, at_warp[PD_WARPS];
        for (int x = first_warp; x <= last_warp; ++x)
          if (b0 + (b1 - b0) * x / PD_WARPS < b0 + (b1 - b0) * (x + 1) / PD_WARPS) at_warp[count++] = x;
        auto at = [&](int i) { return warp_parts + (share * PD_WARPS + at_warp[i]) * 2 + (i == 0 ? first_end : 0); };
        const int in_head = (g % p.chunks) * 8 * NT, head0 = (g / p.chunks) * heads_all + in_head, hn = min(heads_all - in_head, 8 * NT);
        const int64_t r = view_seq(a, s).row;
        auto emit = [&](int h, int c, float o0, float o1, float m, float l) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.o) + r * a.o_stride + (head0 + h) * DH + c) = pack_16<F16>(o0 * inv, o1 * inv);
          if (c == 0 && a.lse) a.lse[r * a.n_q_heads + head0 + h] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
        };
        if (lo >= b0 && hi <= b1) {
          join_parts<DH, 8 * NT>(count, hn, at, emit);
          return;
        }
        Part* mine = share_parts + share * 2 + (lo >= b0 ? 1 : 0);
        join_parts<DH, 8 * NT>(count, hn, at, [&](int h, int c, float o0, float o1, float m, float l) {
          __stcg(reinterpret_cast<float2*>(&mine->o[h][c]), make_float2(o0, o1));
          if (c == 0) __stcg(&mine->ml[h], make_float2(m, l));
        });
        const int f = share_of(lo), e = share_of(hi - 1);
        __threadfence();
        __syncthreads();
        if (tid == 0) {
          const int before = atomicAdd(done_words + f, 1);
          *flag = before == e - f;
          if (before == e - f) done_words[f] = 0;        // ready for the next call
        }
        __syncthreads();
        if (*flag) {
          __threadfence();
          join_parts<DH, 8 * NT>(e - f + 1, hn, [&](int i) { return share_parts + (f + i) * 2 + (i == 0 ? 1 : 0); }, emit);
        }
        __syncthreads();
      };
      int64_t lo, hi;
      int s, g;
      if (c0 == b0) {
        group_at(c0, lo, hi, s, g);
        if (lo < c0) join_run(w, 0, lo, hi, s, g);
      }
      group_at(c1 - 1, lo, hi, s, g);
      if (lo >= c0 && hi > c1) join_run(w, 1, lo, hi, s, g);
      ++w;
    }
    fence_proxy_async();
    __syncthreads();
  }
  if (*abort_flag) drain_after_abort();
}

template <int DH>
constexpr int pd_smem() {
  return 1024 + PD_RING_BYTES + PD_WARPS * PageGeom<DH>::SLOTS * 8 + 64 * 4 + (HS_DEVICE_MAX_SEQS + 1) * 4;
}
static_assert(pd_smem<64>() <= 227 * 1024 && pd_smem<128>() <= 227 * 1024, "fits one SM");
static_assert(size_t(kMaxShares) * (PD_WARPS + 1) * 2 * sizeof(PartOf<128, 16>) <= kWsScratchBytes, "parts of warps and shares");
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
  const int grid = std::min(p.shares, sm_budget);
  return launch_step_kernel(pick(a.head_dim, two, a.type == HS_TYPE_F16, a.cap > 0.f || a.slopes != nullptr), grid, PD_THREADS,
                            a.head_dim == 128 ? pd_smem<128>() : pd_smem<64>(), stream, true, p);
}

}  // namespace hs
