// Attention of one new token per sequence over the paged cache, where the sequences of a group share their first keys, on the 5th-generation
// tensor cores; planned on the device.
//
//   tile      sequences of one group that follow one another, all query heads of one KV head: up to 128 rows of a matrix, sequence after sequence.  Where groups
//             are small (a rule on the call's shape) a tile is 64 rows, which stand in the matrix twice: each copy's softmax has half of a block's keys.
//   keys      the tile's keys are one line of blocks of 64: the group's shared pages, read once for all rows, then the pages of each sequence's own keys, one sequence
//             behind the other, a block of the first half of the rows and one of the second half in turn: they are different warps' work, which overlaps.  A row sees the
//             shared keys and a run of the others; what it does not see is masked, and a warp whose 32 rows see nothing of a block gives it the weight 0 and goes on.  (The products with rows that see nothing cost little: a block's two products take a third of
//             the time that its 32 KB take to come.)
//   teams     two to a thread block, each with a running softmax of its own: a warp that fetches, one that issues S = Q K^T into tensor memory and O += P V, four with one
//             thread per row.  K and V come by 16-byte asynchronous copies: a page's 4 KB are too small a box for the tensor copies, 16 of which a block took
//             1400 cycles.  V rows that no row sees are filled with zeros by the copy.
//   shares    all tiles' lines, one after the other, are cut into equal shares, about one per SM of the device, wherever the cut falls, and each share into halves for
//             the teams.  Both teams come last to the tile in the middle: their rows meet in shared memory, where all eight warps add them up.  A tile that is cut between shares leaves its
//             parts in the workspace; the block that delivers the last one joins them, in order.  Where the cuts lie depends on the lengths and the device,
//             never on the budget, and a block takes one share after the other.
//
// Every block plans for itself, from the lengths, in shared memory.  The softmax works through a block 32 keys at a time in rolled loops, as it is few warps' instructions
// that have to be fetched: unrolled over 64 keys with all its variants the same work took twice as long.
//
// 64 groups of 8 sequences behind 512 .. 2,048 shared keys, 28 heads on 4 of 128, capped: 88 us against a floor of 44 for the bytes; 256 sequences behind 8,191 shared keys with up
// to 1,024 own ones: 123 against 47.  The softmax warps bound the shared keys (1,000 cycles a block of 64 keys for two teams), a row's exponentials and the way of P; own keys
// keep one or two warps of four busy (2,000 cycles).  Plan and first pages are 6 us of a call, the ends and joins of cut tiles 8 to 10.  One group of 4 behind 500 keys: 18.8 us, all latency.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged_tiles.cuh"

namespace hs {
namespace {

constexpr int SA_THREADS = 384, SA_KEYS = 64, SA_ROWS = 128, SA_MAX_SEQS = HS_SHARED_MAX_SEQS;
constexpr int SA_TMEM = 512, SA_TEAM_TMEM = 256;         // columns: of a team, S (two buffers of 64, P over their first 32) and O
constexpr int SA_ITEM_COST = 3;                          // blocks that take as long as a tile's beginning and end
constexpr int SA_MIN_SHARE = 4, SA_MIN_PART = 1;         // blocks, with the tiles' costs; blocks of a part
constexpr int SA_ALONE = 4;                              // rows of a sequence that are worked out together where that has to be done by themselves
constexpr float kRefSlack = 8.f;                         // log2 units by which a row's running maximum may exceed its reference
constexpr float kLn2 = 0.6931471805599453f;

struct SharedParams {
  CUtensorMap tm_q;
  hs_shared_attention_t a;
  ScoreScale score;
  int heads, chunks;                                     // query heads of a tile; groups of them per KV head
  int half_seqs;                                         // of them, the first half: those that begin in the first half of the rows
  int tile_seqs, copies;                                 // sequences of a tile; how often its rows stand in the matrix: 1 or 2
  int shares;                                            // at most
};

// A tile's part in the workspace: outputs relative to the row's reference, four coordinates of all rows after one another, then (reference in log2 units, sum).
template <int DH>
struct RowsPart {
  float4 o[DH / 4][SA_ROWS];
  float2 ml[SA_ROWS];
};

// One item -- a tile, or the part of it that a team has -- the same in every role.
struct Item {
  int valid;
  int seq0, n_seq;                                       // the tile's sequences
  int hk, head0, heads;                                  // KV head, first query head, query heads
  int table;                                             // the sequence whose block table row has the shared pages
  int shared_pages, shared_blocks;
  int block0, n_blocks;                                  // of the tile's line
  int parts, slot;                                       // parts of the tile (1: not cut), and where this one goes
  int middle;                                            // the other team has a part of this part
  int first_b, pages_a, pages_b;                         // own keys: the first sequence of the second half; pages of either half
  int number;                                   // of the tile and its head, in the line
  int begin[SA_ROWS + 1];                                // own pages in front of each sequence's
  int kv[SA_ROWS];                                       // keys of each sequence
  // Block `own` of the own keys: which half it is of (its return value), and its number there; a number behind the half's last page is a block without pages.
  __device__ __forceinline__ int half_of(int own, int& block) const {
    const int a = (pages_a + 3) / 4, b = (pages_b + 3) / 4, both = 2 * min(a, b);
    block = own < both ? own >> 1 : own - min(a, b);
    return own < both ? own & 1 : a < b ? 1 : 0;
  }
};
struct alignas(16) Team {
  uint64_t q_full, q_empty, k_full[2], v_full[2], s_full[2], p_full[2], o_full[2];
  uint64_t ring_full[2], ring_empty[2], end;
  float2 ml[SA_ROWS];                                    // (reference, sum) of rows, at an item's end
  Item ring[2];
};
struct alignas(16) Block {
  uint32_t tmem_base;
  int abort_flag, n_joins;
  int again;                                             // a row that this block has delivered is infinite or NaN
  int middle[2];                                         // whether the teams' last item is the same, in shares of either parity
  int warp_sum[SA_THREADS / 32];
  int joins[kMaxShares];                                 // tiles that this block joins
};

template <int DH>
struct SharedGeom {
  static constexpr int HALVES = DH / 64;
  static constexpr int Q_BYTES = HALVES * 16384;         // [half][128 rows][128 B]
  static constexpr int KV_BYTES = HALVES * 8192;         // K (or V) of a block: [half][4 pages][16 keys][128 B]
  static constexpr int TEAM_BYTES = Q_BYTES + 4 * KV_BYTES;        // Q, two K blocks, two V blocks
  static constexpr int COPY_ROWS = 512 / (DH * 2), COPIES = HS_PAGE_SIZE / COPY_ROWS;        // keys that a warp copies at a time; times for a page
  static constexpr int O0 = 128;                         // of a team's tensor-memory columns
  static constexpr int TEAMS = 2 * TEAM_BYTES, BLOCK = TEAMS + 2 * int(sizeof(Team)), PLAN = BLOCK + int(sizeof(Block));
  // the plan: costs of tiles (running sums), shared pages of groups; first sequences and tiles of groups in 16 bits
  static constexpr int SMEM = 1024 + PLAN + (SA_MAX_SEQS + 2) * (4 + 4 + 2 + 2);
};
static_assert(sizeof(Team) % 16 == 0 && sizeof(Block) % 16 == 0 && SharedGeom<128>::SMEM <= 227 * 1024, "fits one SM");
static_assert(size_t(kMaxShares) * 2 * sizeof(RowsPart<128>) <= kWsScratchBytes, "two parts per share");
static_assert(sizeof(RowsPart<128>) <= SharedGeom<128>::TEAM_BYTES && sizeof(RowsPart<64>) <= SharedGeom<64>::TEAM_BYTES, "a team's rows of the tile in the middle");
static_assert(1024 + kMaxShares * SA_ROWS * 4 <= SharedGeom<64>::TEAMS, "weights of a join");
static_assert(kWsSharedQueue + kMaxShares * 4 <= kWsScratch && SA_MAX_SEQS < 65536, "one word per share");

// The largest and the smallest of three (numbers rather than NaN).
__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
__device__ __forceinline__ float min3(float x, float y, float z) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
// 32 lanes x 16 consecutive 32-bit columns, registers -> tensor memory.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Running sums over the whole block of values(0) .. values(n - 1), a run of them a thread: put(i, sum in front of i); returns the sum of all.
template <typename V, typename U>
__device__ __forceinline__ int running_sums(int n, int* warp_sum, V values, U put) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (n + SA_THREADS - 1) / SA_THREADS, i0 = int(threadIdx.x) * per;
  int mine = 0;
  for (int i = i0; i < min(i0 + per, n); ++i) mine += values(i);
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += x;
  }
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  int before = inc - mine, total = 0;
  for (int w = 0; w < SA_THREADS / 32; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
  for (int i = i0; i < min(i0 + per, n); ++i) {
    const int v = values(i);
    put(i, before);
    before += v;
  }
  __syncthreads();
  return total;
}
// The last i in 0 .. n - 1 with begin[i] <= x.
template <typename T>
__device__ __forceinline__ int find_last(const T* begin, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (int(begin[mid]) <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct Plan {
  const int *cost, *shared;                              // [tiles + 1], [groups]
  const uint16_t *group, *tile;                          // [groups + 1]: first sequence, first tile
  int tiles, line, shares, units;                        // units: KV heads, or chunks of their query heads
  int base, more;                                        // of the line for a share; shares with one more, the first ones
  // An item's number is tile * units + unit; its place in the line is the sum of the costs in front of it.
  __device__ __forceinline__ int blocks_of(int number) const { return cost[number / units + 1] - cost[number / units] - SA_ITEM_COST; }
  __device__ __forceinline__ int place_of(int number) const {
    const int t = number / units;
    return cost[t] * units + (number - t * units) * (cost[t + 1] - cost[t]);
  }
  __device__ __forceinline__ int share_begin(int k) const { return base * k + min(k, more); }
  __device__ __forceinline__ int number_at(int x) const {           // of the item that has place x of the line
    const int t = find_last(cost, tiles, x / units);
    return t * units + (x - cost[t] * units) / (cost[t + 1] - cost[t]);
  }
  // The block of an item in front of which the cut at place x falls; not so near an end that a part would be too short.
  __device__ __forceinline__ int cut_block(int place, int blocks, int x) const {
    const int b = x - place - SA_ITEM_COST;
    return b < SA_MIN_PART ? 0 : b > blocks - SA_MIN_PART ? blocks : b;
  }
  __device__ __forceinline__ int first_share(int x) const {         // the share that has place x
    const int x_more = more * (base + 1);
    return x < x_more ? x / (base + 1) : more + (x - x_more) / base;
  }
};

// The sum of a row's 32 coordinates.
__device__ __forceinline__ float sum_of(const float (&x)[32]) {
  F2 y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = add2(f2(x[4 * e], x[4 * e + 1]), f2(x[4 * e + 2], x[4 * e + 3]));
#pragma unroll
  for (int n = 4; n > 0; n >>= 1)
#pragma unroll
    for (int e = 0; e < n; ++e) y[e] = add2(y[e], y[e + n]);
  float a, b;
  split(y[0], a, b);
  return a + b;
}
// o of a sequence's rows by themselves, by a warp: query heads head .. head + n_heads - 1 (of one KV head, 4 at most), written where `which` has a bit.  32 keys at a time: DH / 8 lanes read
// a key, 16 bytes each, and add up their products; the lane whose turn a key is keeps its scores, weights and place.
template <int DH, bool F16>
__device__ __noinline__ void rows_alone(const SharedParams& p, int seq, int head, int n_heads, unsigned which, int table, int shared_pages) {
  constexpr int H = SA_ALONE, LANES = DH / 8, KEYS = 32 / LANES;
  const hs_shared_attention_t& a = p.a;
  const int lane = threadIdx.x & 31, pos = lane % LANES, sub = lane / LANES, lane0 = lane - pos;
  const int kv = min(max(a.kv_len[seq], 0), row_tokens(a.max_pages_per_seq)), hk = head / (a.n_q_heads / a.n_kv_heads);
  const uint16_t* pool = static_cast<const uint16_t*>(a.kv_pool) + ((int64_t(a.layer * 2) * a.num_pages) * a.n_kv_heads + hk) * (HS_PAGE_SIZE * DH) + pos * 8;
  const int64_t to_v = int64_t(a.num_pages) * a.n_kv_heads * (HS_PAGE_SIZE * DH);
  auto unpack = [](const uint4& w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float2 f;
      if constexpr (F16) f = __half22float2(*reinterpret_cast<const __half2*>(&u[e]));
      else f = make_float2(__uint_as_float(u[e] << 16), __uint_as_float(u[e] & 0xffff0000u));
      x[2 * e] = f.x;
      x[2 * e + 1] = f.y;
    }
  };
  float q[H][8], o[H][8] = {}, m[H], l[H] = {}, slope[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int of = head + min(h, n_heads - 1);
    unpack(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + seq * a.q_stride + of * DH + pos * 8), q[h]);
    m[h] = -INFINITY;
    slope[h] = a.slopes ? a.slopes[of] * 1.4426950408889634f : 0.f;
  }
#pragma unroll 1
  for (int j0 = 0; j0 < kv; j0 += 32) {
    const int j = j0 + pos * KEYS + sub, page = j / HS_PAGE_SIZE;
    int64_t at = -1;                                     // of the lane's key among those of the KV head; a page outside the pool has none
    if (j < kv) {
      const int id = a.block_tables[int64_t(page < shared_pages ? table : seq) * a.max_pages_per_seq + page];
      if (id >= 0 && id < a.num_pages) at = int64_t(id) * a.n_kv_heads * (HS_PAGE_SIZE * DH) + (j % HS_PAGE_SIZE) * DH;
    }
    auto each_key = [&](const uint16_t* from, auto use) {          // use(lane of this group that has the key, its 8 coordinates); zeros for no key
#pragma unroll 1
      for (int i0 = 0; i0 < LANES; i0 += 8) {
        uint4 w[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int64_t of = __shfl_sync(0xffffffffu, at, lane0 + i0 + u);
          w[u] = of >= 0 ? *reinterpret_cast<const uint4*>(from + of) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          float x[8];
          unpack(w[u], x);
          use(i0 + u, x);
        }
      }
    };
    float w[H];
    each_key(pool, [&](int i, float(&x)[8]) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(q[h][e], x[e], dot);
#pragma unroll
        for (int n = LANES / 2; n > 0; n >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, n);
        w[h] = pos == i ? dot : i == 0 ? 0.f : w[h];
      }
    });
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float y = p.score.out == 0.f ? w[h] * p.score.in : tanh_any(w[h] * p.score.in) * p.score.out;
      const float x = at >= 0 ? fmaf(-slope[h], float(kv - 1 - j), y) : -INFINITY;
      float top = fmaxf(m[h], x);
#pragma unroll
      for (int n = 16; n > 0; n >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, n));
      const float zero = top == -INFINITY ? 0.f : top, f = fast_exp2(m[h] - zero);
      m[h] = top;
      w[h] = fast_exp2(x - zero);
      l[h] = fmaf(l[h], f, w[h]);                        // (of the lane's keys)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[h][e] *= f;
    }
    each_key(pool + to_v, [&](int i, float(&x)[8]) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const float of = __shfl_sync(0xffffffffu, w[h], lane0 + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[h][e] = fmaf(of, x[e], o[h][e]);
      }
    });
    // (nothing that follows changes rows that are NaN from end to end: those of a whole group, behind such a shared key)
    bool over = true;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) over &= o[h][e] != o[h][e];
    unsigned who = __ballot_sync(0xffffffffu, over);
#pragma unroll
    for (int n = 16; n >= LANES; n >>= 1) who |= who >> n;           // (the lanes that have the same coordinates of other keys)
    if ((~who & ((1u << LANES) - 1u)) == 0) break;
  }
#pragma unroll
  for (int h = 0; h < H; ++h) {
#pragma unroll
    for (int n = 16; n > 0; n >>= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], n);
    const float inv = l[h] == 0.f ? 0.f : 1.f / l[h];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int n = 16; n >= LANES; n >>= 1) o[h][e] += __shfl_xor_sync(0xffffffffu, o[h][e], n);
      o[h][e] *= inv;
    }
    if (sub == 0 && (which >> h & 1u))
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.o) + seq * a.o_stride + (head + h) * DH + pos * 8) =
          make_uint4(pack_16<F16>(o[h][0], o[h][1]), pack_16<F16>(o[h][2], o[h][3]), pack_16<F16>(o[h][4], o[h][5]), pack_16<F16>(o[h][6], o[h][7]));
  }
}

// The weight 0 of a key that a row does not see gives NaN where its v is infinite or NaN.  A block that has finished such a row looks through the tiles that it has finished: rows with
// an output that is no number are worked out once more, a sequence's by themselves.  Those that see such a v keep what it gives.
template <int DH, bool F16>
__device__ __noinline__ void finished_again(const SharedParams& p, const Plan plan, const int* joins, int n_joins) {
  const hs_shared_attention_t& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, heads_all = a.n_q_heads / a.n_kv_heads;
  auto tile_again = [&](int number) {
    const int t = number / plan.units, unit = number - t * plan.units, g = find_last(plan.tile, a.n_groups, t), g_end = plan.group[g + 1];
    const int s0 = int(plan.group[g]) + (t - int(plan.tile[g])) * p.tile_seqs, n = min(g_end - s0, p.tile_seqs);
    const int hk = unit / p.chunks, in_head = (unit - hk * p.chunks) * p.heads, heads = min(heads_all - in_head, p.heads);
    int table = plan.group[g];                           // (one of the group's has keys, where there are shared pages)
    while (plan.shared[g] > 0 && table < g_end - 1 && a.kv_len[table] <= 0) ++table;
    const int fours = (heads + SA_ALONE - 1) / SA_ALONE;
#pragma unroll 1
    for (int i = warp; i < n * fours; i += SA_THREADS / 32) {
      const int seq = s0 + i / fours, in_tile = i % fours * SA_ALONE, head = hk * heads_all + in_head + in_tile, n_heads = min(heads - in_tile, SA_ALONE);
      constexpr int kExponent = F16 ? 0x7c00 : 0x7f80;
      unsigned which = 0;
      for (int h = 0; h < n_heads; ++h) {
        const uint16_t* row = static_cast<const uint16_t*>(a.o) + seq * a.o_stride + (head + h) * DH;
        bool bad = false;
        for (int c = lane; c < DH; c += 32) bad |= (row[c] & kExponent) == kExponent;
        which |= __any_sync(0xffffffffu, bad) ? 1u << h : 0u;
      }
      if (which) rows_alone<DH, F16>(p, seq, head, n_heads, which, table, plan.shared[g]);
    }
  };
#pragma unroll 1
  for (int share = int(blockIdx.x); share < plan.shares; share += int(gridDim.x)) {
    const int x0 = plan.share_begin(share), x1 = plan.share_begin(share + 1), last = plan.number_at(x1 - 1);
#pragma unroll 1
    for (int number = plan.number_at(x0); number <= last; ++number) {
      const int place = plan.place_of(number), blocks = plan.blocks_of(number);
      const int from = place < x0 ? plan.cut_block(place, blocks, x0) : 0, to = place + blocks + SA_ITEM_COST > x1 ? plan.cut_block(place, blocks, x1) : blocks;
      if (from == 0 && to == blocks) tile_again(number);
    }
  }
#pragma unroll 1
  for (int i = 0; i < n_joins; ++i) tile_again(joins[i]);
}

template <int DH, bool F16, bool MOD>
__global__ void __launch_bounds__(SA_THREADS, 1) shared_attention_kernel(const __grid_constant__ SharedParams p) {
  using G_ = SharedGeom<DH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Block* bar = reinterpret_cast<Block*>(smem + G_::BLOCK);
  volatile int* abort_flag = &bar->abort_flag;
  const hs_shared_attention_t& a = p.a;
  // (the warp's number by a shuffle, so that the compiler knows it is the same in all lanes: descriptors then stay in uniform registers)
  const int warp = __shfl_sync(0xffffffffu, int(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31, tid = int(threadIdx.x);
  // Warps 0 .. 3 and 4 .. 7 are the teams' softmax warps (of tensor memory lanes 32 (warp % 4) on), 8 and 10 fetch, 9 and 11 issue the products.
  const int team = warp < 8 ? warp >> 2 : (warp - 8) >> 1;
  Team& tm = reinterpret_cast<Team*>(smem + G_::TEAMS)[team];
  uint8_t* q_smem = smem + team * G_::TEAM_BYTES;
  uint8_t* k_smem = q_smem + G_::Q_BYTES;
  uint8_t* v_smem = k_smem + 2 * G_::KV_BYTES;
  const int n_seqs = a.n_seqs, n_groups = a.n_groups, units = a.n_kv_heads * p.chunks;
  const int most_keys = row_tokens(a.max_pages_per_seq);

  if (tid < 2) {
    Team& t = reinterpret_cast<Team*>(smem + G_::TEAMS)[tid];
    mbar_init(&t.q_full, 1);
    mbar_init(&t.q_empty, 4);                            // one arrival per softmax warp, here and below
    for (int i = 0; i < 2; ++i) {
      mbar_init(&t.k_full[i], 32);                       // one per lane of the warp that fetches, behind its copies
      mbar_init(&t.v_full[i], 32);
      mbar_init(&t.s_full[i], 1);
      mbar_init(&t.p_full[i], 4);
      mbar_init(&t.o_full[i], 1);
      mbar_init(&t.ring_full[i], 1);
      mbar_init(&t.ring_empty[i], 5);                    // four softmax warps and the one that issues products
    }
    mbar_init(&t.end, 4);
    fence_barrier_init();
  }
  if (tid == 0) {
    bar->abort_flag = 0;
    bar->n_joins = 0;
    bar->again = 0;
    tma_prefetch_desc(&p.tm_q);
  }
  if (warp == 9) {
    tmem_alloc(&bar->tmem_base, SA_TMEM);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = bar->tmem_base;
  griddep_wait();

  // ---------------------------------------------------------------- the plan
  auto keys_of = [&](int s) { return min(max(a.kv_len[s], 0), most_keys); };
  Plan plan;
  {
    int* cost = reinterpret_cast<int*>(smem + G_::PLAN);
    int* shared = cost + SA_MAX_SEQS + 2;
    uint16_t* group = reinterpret_cast<uint16_t*>(shared + SA_MAX_SEQS + 2);
    uint16_t* tile = group + SA_MAX_SEQS + 2;
    // (a thread's first sequences: their lengths are asked for before the groups are known, and kept)
    constexpr int MINE = 2;
    int kv[MINE], of[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) kv[i] = tid + i * SA_THREADS < n_seqs ? a.kv_len[tid + i * SA_THREADS] : 0;
    int wrong = 0;
    for (int g = tid; g <= n_groups; g += SA_THREADS) {
      const int b = a.group_begin[g];
      wrong |= b < 0 || b > n_seqs || (g < n_groups && (a.group_begin[g + 1] < b || a.shared_len[g] < 0));
      group[g] = uint16_t(b);
      shared[g] = 0x7fffffff;                            // (the fewest keys of a sequence that has some)
    }
    for (int t = tid; t < n_seqs; t += SA_THREADS) cost[t] = 0;
    wrong = __syncthreads_or(wrong);
    if (wrong) {
      if (tid == 0 && blockIdx.x == 0) atomicExch(a.status, kErrInvalidArg);
      if (warp == 9) tmem_dealloc(tmem, SA_TMEM);
      return;
    }
    const int s_begin = group[0], s_end = group[n_groups];
    // every sequence of a group: its keys and its group
    auto each = [&](auto use) {
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const int s = tid + i * SA_THREADS;
        if (s >= s_begin && s < s_end && kv[i] > 0) use(s, kv[i], of[i]);
      }
      for (int s = tid + MINE * SA_THREADS; s < s_end; s += SA_THREADS) {
        const int keys = s >= s_begin ? keys_of(s) : 0;
        if (keys > 0) use(s, keys, find_last(group, n_groups, s));
      }
    };
    int bad = 0;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int s = tid + i * SA_THREADS;
      if (s < s_begin || s >= s_end) continue;
      bad |= kv[i] < 0 || kv[i] > most_keys;
      kv[i] = min(max(kv[i], 0), most_keys);
      of[i] = find_last(group, n_groups, s);
    }
    if (blockIdx.x == 0) {
      for (int s = tid + MINE * SA_THREADS; s < s_end; s += SA_THREADS) bad |= s >= s_begin && (a.kv_len[s] < 0 || a.kv_len[s] > most_keys);
      if (bad) atomicExch(a.status, kErrBadBlockTable);
    }
    each([&](int, int keys, int g) { atomicMin(&shared[g], keys); });
    plan.tiles = running_sums(n_groups, bar->warp_sum, [&](int g) { return (int(group[g + 1]) - int(group[g]) + p.tile_seqs - 1) / p.tile_seqs; },
                              [&](int g, int sum) {
                                tile[g] = uint16_t(sum);
                                shared[g] = shared[g] == 0x7fffffff ? 0 : min(shared[g], a.shared_len[g]) / HS_PAGE_SIZE;
                              });
    if (tid == 0) tile[n_groups] = uint16_t(plan.tiles);
    each([&](int s, int keys, int g) {
      atomicAdd(&cost[int(tile[g]) + (s - int(group[g])) / p.tile_seqs], (keys + HS_PAGE_SIZE - 1) / HS_PAGE_SIZE - shared[g]);
    });
    __syncthreads();
    // (at least one block, so that rows that see no key take the same way, too)
    const int all = running_sums(plan.tiles, bar->warp_sum,
                                 [&](int t) {
                                   const int g = t < n_groups && tile[t] == t && tile[t + 1] > t ? t : find_last(tile, n_groups, t);
                                   // (with sequences in both halves there may be one block more)
                                   const int two = int(group[g + 1]) - int(group[g]) - (t - int(tile[g])) * p.tile_seqs > p.half_seqs ? 1 : 0;
                                   return max((shared[g] + 3) / 4 + (cost[t] + 3) / 4 + two, 1) + SA_ITEM_COST;
                                 },
                                 [&](int t, int sum) { cost[t] = sum; });
    if (tid == 0) cost[plan.tiles] = all;
    __syncthreads();
    plan.cost = cost;
    plan.shared = shared;
    plan.group = group;
    plan.tile = tile;
    plan.units = units;
    plan.line = all * units;
    // Small calls: a share's blocks come one after the other, and so do the parts that a join reads, so the shares grow with the root of the tiles' lengths.  Measured at head_dim 128
    // with three sets of inputs in turn, against shares of 6 blocks and parts of 2 or more for every length: 4 sequences behind 500 keys, 28 heads on 4, 19.4 us for 21.3; one behind
    // 32,000, 7 on one, 43.8 for 68.2; 8 behind 16,000, 14 on two, 34.1 for 43.3.
    const int least = max(SA_MIN_SHARE, int(sqrtf(float(all) / float(max(plan.tiles, 1)))));
    plan.shares = max(1, min(p.shares, plan.line / least));
    plan.base = plan.line / plan.shares;
    plan.more = plan.line - plan.base * plan.shares;
  }
  // Whether both teams have blocks of the item in their share.
  auto middle_of = [&](int share, int number) {
    const int x0 = plan.share_begin(share), x1 = plan.share_begin(share + 1), xm = x0 + (x1 - x0) / 2, place = plan.place_of(number), blocks = plan.blocks_of(number);
    const int end = place + blocks + SA_ITEM_COST;
    if (place >= xm || end <= xm) return 0;
    const int from = place < x0 ? plan.cut_block(place, blocks, x0) : 0, at = plan.cut_block(place, blocks, xm), to = end > x1 ? plan.cut_block(place, blocks, x1) : blocks;
    return from < at && at < to ? 1 : 0;
  };

  // The shares' parts of an item: block ranges between the cuts that fall into it; how many there are (a warp asks).
  auto count_parts = [&](int number, int place, int blocks) {
    const int end = place + blocks + SA_ITEM_COST, f = plan.first_share(place);
    int parts = 0;
    for (int k0 = f; k0 < plan.shares && plan.share_begin(k0) < end; k0 += 32) {
      const int k = k0 + lane;
      bool has = false;
      if (k < plan.shares && plan.share_begin(k) < end) {
        const int from = k == f ? 0 : plan.cut_block(place, blocks, plan.share_begin(k));
        has = from < (plan.share_begin(k + 1) < end ? plan.cut_block(place, blocks, plan.share_begin(k + 1)) : blocks);
      }
      parts += __popc(__ballot_sync(0xffffffffu, has));
    }
    return parts;
  };

  auto warp_wait = [&](uint64_t* b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, a.status)) != 0; };
  int rs = 0;
  uint32_t rph = 0;                                      // item ring slot / phase
  uint32_t items_seen = 0;
  uint32_t g = 0;                                        // blocks of this team's earlier items
  float m_ref = -INFINITY, l_run = 0.f;                  // softmax: of a row (MOD: in log2 units; else of the raw scores, whose scale is positive)
  const int copies = p.copies, copy_rows = SA_ROWS / copies;
  uint32_t sreg[32];                                     // softmax: 32 scores, or 32 columns of O

  // The rows' outputs of an item that has ended, 32 columns at a time: from tensor memory, scaled by f, the other copy's added to the first copy's.
  // use(columns' place, values) is called by the threads of the first copy.  Returns false where a wait has given up.
  const int r = tid & 127;                               // row of the matrix = lane of tensor memory
  const uint32_t t_lane = tmem + team * SA_TEAM_TMEM + (uint32_t((warp & 3) * 32) << 16);
  uint32_t end_phase = 0;
  auto team_wait = [&]() {                               // the team's softmax warps
    __syncwarp();
    if (lane == 0) mbar_arrive(&tm.end);
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&tm.end, end_phase, abort_flag, a.status));
    end_phase ^= 1;
    return ok;
  };
  auto row_reference = [&]() { return m_ref == -INFINITY ? -INFINITY : MOD ? m_ref : __fmul_rn(m_ref, p.score.in); };          // in log2 units
  // (reference, sum) of the thread's row over its copies; f: what the thread's own outputs count
  auto row_total = [&](float& f, bool& ok) {
    const float m_log2 = row_reference();
    f = 1.f;
    ok = true;
    if (copies == 1) return make_float2(m_log2, l_run);
    tm.ml[r] = make_float2(m_log2, l_run);
    ok = team_wait();
    const float2 x = tm.ml[r & 63], y = tm.ml[(r & 63) + 64];
    const float top = fmaxf(x.x, y.x), zero = top == -INFINITY ? 0.f : top;
    f = fast_exp2(m_log2 - zero);
    return make_float2(top, fmaf(x.y, fast_exp2(x.x - zero), y.y * fast_exp2(y.x - zero)));
  };
  auto each_columns = [&](float f, auto use) {
    float4* other = reinterpret_cast<float4*>(q_smem);   // [columns / 4][64 rows]: the second copy's rows (Q is read no more)
    bool ok = true;
    if (copies == 2 && r >= 64) {
#pragma unroll 1
      for (int c = 0; c < DH; c += 32) {
        tmem_ld32(t_lane + G_::O0 + c, sreg);
        tmem_ld_wait();
#pragma unroll
        for (int u = 0; u < 8; ++u)
          other[(c / 4 + u) * 64 + r - 64] = make_float4(__uint_as_float(sreg[4 * u]) * f, __uint_as_float(sreg[4 * u + 1]) * f, __uint_as_float(sreg[4 * u + 2]) * f,
                                                         __uint_as_float(sreg[4 * u + 3]) * f);
      }
    }
    if (copies == 2) ok = team_wait();
    if (copies == 1 || r < 64) {
#pragma unroll 1
      for (int c = 0; c < DH; c += 32) {
        tmem_ld32(t_lane + G_::O0 + c, sreg);
        tmem_ld_wait();
        float x[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(sreg[e]) * f;
        if (copies == 2) {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const float4 y = other[(c / 4 + u) * 64 + r];
            x[4 * u] += y.x;
            x[4 * u + 1] += y.y;
            x[4 * u + 2] += y.z;
            x[4 * u + 3] += y.w;
          }
        }
        use(c, x);
      }
    }
    return ok;
  };
  // Finished rows, or a part of them in the workspace.
  auto deliver = [&](const Item& it, float2 total, float f) {
    const int row_in = copies == 2 ? r & 63 : r, i_seq = row_in / p.heads, h = row_in - i_seq * p.heads;
    const bool mine = r < copy_rows && i_seq < it.n_seq && h < it.heads;
    const int64_t row = it.seq0 + i_seq;
    const int head = it.head0 + h;
    const float inv = total.y == 0.f ? 0.f : 1.f / total.y;
    uint16_t* dst = static_cast<uint16_t*>(a.o) + row * a.o_stride + head * DH;
    RowsPart<DH>& part = reinterpret_cast<RowsPart<DH>*>(static_cast<char*>(a.workspace) + kWsScratch)[it.slot];
    const bool whole = it.parts == 1;
    if (mine) {
      if (!whole) __stcg(&part.ml[r], total);
      else if (a.lse) a.lse[row * a.n_q_heads + head] = total.y == 0.f ? -INFINITY : kLn2 * (total.x + log2f(total.y));
    }
    float none = 0.f;                                    // NaN where an output is infinite or NaN
    const bool ok = each_columns(f, [&](int c, float(&x)[32]) {
      if (!mine) return;
      if (whole) {
        none = fmaf(sum_of(x), 0.f, none);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          *reinterpret_cast<uint4*>(dst + c + u * 8) = make_uint4(pack_16<F16>(x[8 * u] * inv, x[8 * u + 1] * inv), pack_16<F16>(x[8 * u + 2] * inv, x[8 * u + 3] * inv),
                                                                  pack_16<F16>(x[8 * u + 4] * inv, x[8 * u + 5] * inv), pack_16<F16>(x[8 * u + 6] * inv, x[8 * u + 7] * inv));
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) __stcg(&part.o[c / 4 + u][r], make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]));
      }
    });
    if (none != 0.f && total.y < INFINITY) bar->again = 1;          // (a row whose sum is NaN has a q or k that is)
    return ok;
  };
  // A part of an item with so many has arrived, by one of its four warps (n = 1) or all of it (n = 4).
  auto arrived = [&](int number, int parts, int n) {
    int* done = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsSharedQueue) + plan.first_share(plan.place_of(number));
    if (atomicAdd(done, n) == 4 * parts - n) {
      *done = 0;                                         // ready for the next call
      bar->joins[atomicAdd(&bar->n_joins, 1)] = number;
    }
  };

#pragma unroll 1
  for (int share = plan.tiles > 0 ? int(blockIdx.x) : plan.shares, turn = 0; share < plan.shares; share += int(gridDim.x), ++turn) {
    const int x0 = plan.share_begin(share), x1 = plan.share_begin(share + 1), xm = x0 + (x1 - x0) / 2;
    int middle = 0;                                      // softmax: of the last item
    if (warp == 8 || warp == 10) {
      // ============================================================ fetching ==
      // Items from this team's half of the share, the first team's in rising order, the second's in falling order, so that both come to the middle last.
      // A copy of a warp is 512 bytes: COPY_ROWS keys of a page.  This lane's 16 bytes are chunk (lane % chunks of a key) of key lane / chunks of each; they go where
      // the 128-byte swizzle has them: chunk c of key r of a 64-coordinate half at r * 128 + ((c ^ r % 8) * 16).
      constexpr int CHUNKS = DH / 8;
      const int chunk = lane % CHUNKS, key = lane / CHUNKS;
      const int64_t page_bytes = int64_t(a.n_kv_heads) * (HS_PAGE_SIZE * DH * 2);
      const uint32_t to = uint32_t((chunk >> 3) * 8192 + key * 128 + (((chunk & 7) ^ key) << 4));
      const int xa = team == 0 ? x0 : xm, xb = team == 0 ? xm : x1;
      const int first = xa < xb ? plan.number_at(xa) : 0, last = xa < xb ? plan.number_at(xb - 1) : -1;
      bool ok = true;
      int t_cached = -1;                                 // the tile whose sequences are in the ring's other slot
      for (int i = 0; ok; ++i) {
        // the next item that has blocks
        int number = 0, t = 0, unit = 0, place = 0, blocks = 0, b0 = 0, b1 = 0;
        bool some = false;
        for (; i <= last - first && !some; ++i) {
          number = team == 0 ? first + i : last - i;
          t = number / units;
          unit = number - t * units;
          blocks = plan.cost[t + 1] - plan.cost[t] - SA_ITEM_COST;
          place = plan.cost[t] * units + unit * (blocks + SA_ITEM_COST);
          b0 = place < xa ? plan.cut_block(place, blocks, xa) : 0;
          b1 = place + blocks + SA_ITEM_COST > xb ? plan.cut_block(place, blocks, xb) : blocks;
          some = b0 < b1;
        }
        --i;
        if (lane == 0) ok = mbar_wait(&tm.ring_empty[rs], rph ^ 1, abort_flag, a.status);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        Item& it = tm.ring[rs];
        if (!some) {
          if (lane == 0) {
            it.valid = 0;
            mbar_arrive(&tm.ring_full[rs]);
          }
          if (++rs == 2) { rs = 0; rph ^= 1; }
          break;
        }
        {
          const int grp = find_last(plan.tile, n_groups, t);
          const int g_begin = plan.group[grp], g_end = plan.group[grp + 1], s0 = g_begin + (t - int(plan.tile[grp])) * p.tile_seqs, n = min(g_end - s0, p.tile_seqs);
          const int shared_pages = plan.shared[grp];
          int table = g_begin, sum = 0;
          if (t == t_cached) {                           // the other slot has the same tile of another head
            const Item& prev = tm.ring[rs ^ 1];
            for (int k = lane; k < n; k += 32) {
              it.begin[k] = prev.begin[k];
              it.kv[k] = prev.kv[k];
            }
            table = prev.table;
            sum = prev.begin[n];
          } else {
            if (shared_pages > 0) {
              for (int s = g_begin; s < g_end; s += 32) {          // (one of the group's has keys)
                const unsigned who = __ballot_sync(0xffffffffu, s + lane < g_end && keys_of(s + lane) > 0);
                if (who) {
                  table = s + __ffs(who) - 1;
                  break;
                }
              }
            }
            for (int k = 0; k < n; k += 32) {
              const int keys = k + lane < n ? keys_of(s0 + k + lane) : 0;
              const int pages = keys > 0 ? (keys + HS_PAGE_SIZE - 1) / HS_PAGE_SIZE - shared_pages : 0;
              int inc = pages;
#pragma unroll
              for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += x;
              }
              if (k + lane < n) {
                it.begin[k + lane] = sum + inc - pages;
                it.kv[k + lane] = keys;
              }
              sum += __shfl_sync(0xffffffffu, inc, 31);
            }
            t_cached = t;
          }
          const int parts = count_parts(number, place, blocks);
          if (lane == 0) {
            it.valid = 1;
            it.seq0 = s0;
            it.n_seq = n;
            it.hk = unit / p.chunks;
            const int in_head = (unit - it.hk * p.chunks) * p.heads, heads_all = a.n_q_heads / a.n_kv_heads;
            it.head0 = it.hk * heads_all + in_head;
            it.heads = min(heads_all - in_head, p.heads);
            it.table = table;
            it.shared_pages = shared_pages;
            it.shared_blocks = (shared_pages + 3) / 4;
            it.block0 = b0;
            it.n_blocks = b1 - b0;
            it.parts = parts;
            it.slot = 2 * share + (place < x0 ? 0 : 1);
            it.middle = middle_of(share, number);
            it.number = number;
            it.begin[n] = sum;
            it.first_b = min(p.half_seqs, n);
          }
          __syncwarp();
          if (lane == 0) {
            it.pages_a = it.begin[it.first_b];
            it.pages_b = sum - it.pages_a;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&tm.ring_full[rs]);
        const int n_seq = it.n_seq, n_blocks = it.n_blocks, block0 = it.block0, shared_pages = it.shared_pages, shared_blocks = it.shared_blocks;
        // Lane l looks up page l % 4 of block j0 + l / 4: its id and how many of its keys are seen (0: there is no such page).
        int keys = 0;
        auto look_up = [&](int j0) {
          const int j = j0 + (lane >> 2);
          keys = 0;
          if (j >= n_blocks) return 0;
          if (block0 + j < shared_blocks) {
            const int u = (block0 + j) * 4 + (lane & 3);
            if (u >= shared_pages) return 0;
            keys = HS_PAGE_SIZE;
            return a.block_tables[int64_t(it.table) * a.max_pages_per_seq + u];
          }
          int block;
          const int second = it.half_of(block0 + j - shared_blocks, block);
          int u = block * 4 + (lane & 3);
          if (u >= (second ? it.pages_b : it.pages_a)) return 0;
          u += second ? it.pages_a : 0;
          const int k = find_last(it.begin, n_seq, u), page = shared_pages + u - it.begin[k];
          keys = min(it.kv[k] - page * HS_PAGE_SIZE, HS_PAGE_SIZE);
          return a.block_tables[int64_t(it.seq0 + k) * a.max_pages_per_seq + page];
        };
        // An id and its keys in one word (the pool has fewer than 2^26 pages); a page outside the pool has no keys.
        auto checked = [&](int id, int n) {
          if (n > 0 && (id < 0 || id >= a.num_pages)) {
            atomicExch(a.status, kErrBadBlockTable);
            n = 0;
          }
          return n > 0 ? (n << 26) | id : 0;
        };
        const char* pool = static_cast<const char*>(a.kv_pool) + (int64_t(a.layer * 2) * a.num_pages * a.n_kv_heads + it.hk) * (HS_PAGE_SIZE * DH * 2) + lane * 16;
        // The pages of eight blocks: K's, V's where K is ahead of them, and the ids that are on their way for the next eight.
        int k_pages = look_up(0), v_pages = 0, k_eight = 0;
        k_pages = checked(k_pages, keys);
        int raw = look_up(8), raw_keys = keys;
        // K of blocks 0 and 1, then V of a block and K of the one behind the next in turn.
#pragma unroll 1
        for (int e = -2; ok && e < 2 * n_blocks; ++e) {
          const int kv = e >= 0 && (e & 1) == 0 ? 1 : 0, j = e < 0 ? e + 2 : kv ? e >> 1 : (e >> 1) + 2;
          // the Q tile, for which the item in front has to be done with its own, behind the first two K blocks
          if (e == 0) {
            ok = warp_wait(&tm.q_empty, (items_seen & 1) ^ 1);
            if (ok && lane == 0) {
              mbar_expect_tx(&tm.q_full, copies * G_::HALVES * p.heads * p.tile_seqs * 128);
#pragma unroll 1
              for (int k = 0; k < copies; ++k)
#pragma unroll 1
                for (int h = 0; h < G_::HALVES; ++h)
                  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                                   smem_u32(q_smem + h * 16384 + k * 8192)),
                               "l"(reinterpret_cast<uint64_t>(&p.tm_q)), "r"(smem_u32(&tm.q_full)), "r"(h * 64), "r"(it.head0), "r"(it.seq0)
                               : "memory");
            }
            if (!ok) break;
          }
          if (j >= n_blocks) continue;
          if (!kv && (j & 7) == 0 && j > 0) {
            v_pages = k_pages;
            k_pages = checked(raw, raw_keys);
            k_eight = j >> 3;
            raw = look_up(j + 8);
            raw_keys = keys;
          }
          const uint32_t b = g + j, buf = b & 1;
          // a slot is free when the products with what it held are done
          if (b >= 2) ok = warp_wait(kv ? &tm.o_full[buf] : &tm.s_full[buf], ((b - 2) >> 1) & 1);
          if (!ok) break;
          const uint32_t dst = smem_u32((kv ? v_smem : k_smem) + buf * G_::KV_BYTES) + to;
          const char* src_kv = pool + kv * int64_t(a.num_pages) * page_bytes;
          const int pages = j >> 3 == k_eight ? k_pages : v_pages;
#pragma unroll 1
          for (int w = 0; w < 4; ++w) {
            const int word = __shfl_sync(0xffffffffu, pages, (j & 7) * 4 + w), n = word >> 26;
            if (n == 0 && !kv) continue;                 // (scores that no row looks at; V has to be finite everywhere)
            const char* src = src_kv + int64_t(word & ((1 << 26) - 1)) * page_bytes;
#pragma unroll
            for (int c = 0; c < G_::COPIES; ++c)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((dst ^ (((c * G_::COPY_ROWS) & 7) << 4)) + w * 2048 + c * G_::COPY_ROWS * 128),
                           "l"(src + c * 512), "r"(c * G_::COPY_ROWS + key < n ? 16 : 0)
                           : "memory");
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(kv ? &tm.v_full[buf] : &tm.k_full[buf])) : "memory");
        }
        __syncwarp();
        ++items_seen;
        g += n_blocks;
        if (++rs == 2) { rs = 0; rph ^= 1; }
      }
    } else if (warp == 9 || warp == 11) {
      // ============================================================= products ==
      // (the whole warp goes through the loop, and one lane issues: a thread by itself took 77 cycles for each product, to bring its descriptor to uniform registers)
      constexpr uint32_t idesc_s = idesc_16<F16>(128, SA_KEYS);
      constexpr uint32_t idesc_pv = idesc_16<F16>(128, DH) | (1u << 16);     // B (= V) is MN-major
      const uint64_t q_desc = umma_desc_kmajor_sw128(smem_u32(q_smem));
      const uint64_t k_desc0 = umma_desc_kmajor_sw128(smem_u32(k_smem));
      const uint64_t v_desc0 = umma_desc_mnmajor_sw128(smem_u32(v_smem), 8192, 1024);
      const uint32_t s_base = tmem + team * SA_TEAM_TMEM, d_o = s_base + G_::O0;
      bool ok = true;
#pragma unroll 1
      while (ok) {
        ok = warp_wait(&tm.ring_full[rs], rph);
        if (!ok) break;
        const int valid = __shfl_sync(0xffffffffu, tm.ring[rs].valid, 0), n_blocks = __shfl_sync(0xffffffffu, tm.ring[rs].n_blocks, 0);
        if (lane == 0) mbar_arrive(&tm.ring_empty[rs]);
        if (++rs == 2) { rs = 0; rph ^= 1; }
        if (!valid) break;
        ok = warp_wait(&tm.q_full, items_seen & 1);
        ++items_seen;
        // S of block j, then P V of block j - 1, which overlaps the softmax of block j
#pragma unroll 1
        for (int j = 0; j <= n_blocks && ok; ++j) {
          if (j < n_blocks) {
            const uint32_t b = g + j, buf = b & 1;
            ok = warp_wait(&tm.k_full[buf], (b >> 1) & 1);
            if (!ok) break;
            fence_proxy_async();                         // (K came by ordinary copies)
            tc_fence_after_sync();
            const uint64_t kdesc = k_desc0 + uint64_t(buf * (G_::KV_BYTES >> 4));
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < DH / 16; ++ks)
                umma_bf16(s_base + buf * SA_KEYS, q_desc + uint64_t((ks >> 2) * (16384 >> 4) + 2 * (ks & 3)),
                          kdesc + uint64_t((ks >> 2) * (8192 >> 4) + 2 * (ks & 3)), idesc_s, ks != 0);
              umma_commit(&tm.s_full[buf]);              // (which frees the K slot, too)
            }
            __syncwarp();
          }
          if (j > 0) {
            const uint32_t b = g + j - 1, buf = b & 1, ph = (b >> 1) & 1;
            ok = warp_wait(&tm.v_full[buf], ph) && warp_wait(&tm.p_full[buf], ph);
            if (!ok) break;
            fence_proxy_async();                         // (V came by ordinary copies)
            tc_fence_after_sync();
            const uint64_t vdesc = v_desc0 + uint64_t(buf * (G_::KV_BYTES >> 4));
            if (elect_one()) {
#pragma unroll
              for (int pg = 0; pg < 4; ++pg)             // 16 keys (one page) per MMA: 8 columns of P; the item's first block overwrites O
                umma_ts(d_o, s_base + buf * SA_KEYS + 8 * pg, vdesc + uint64_t(pg * (2048 >> 4)), idesc_pv, pg != 0 || j != 1 ? 1u : 0u);
              umma_commit(&tm.o_full[buf]);              // (which frees the V slot, too)
            }
            __syncwarp();
          }
        }
        g += n_blocks;
      }
    } else {
      // ============================================================== softmax ==
      const ScoreScale& sc = p.score;
      const int row_in = copies == 2 ? r & 63 : r, i_seq = row_in / p.heads, h = row_in - i_seq * p.heads;      // (rows of a box have room for p.heads each)
      const int n_chunks = copies == 2 ? 1 : 2, half = copies == 2 && r >= 64 ? 1 : 0;     // 32 keys at a time: how many times, and the first
      for (;;) {
        bool ok = __all_sync(0xffffffffu, mbar_wait(&tm.ring_full[rs], rph, abort_flag, a.status));
        if (!ok) break;
        const Item& it = tm.ring[rs];
        if (!it.valid) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&tm.ring_empty[rs]);
          if (++rs == 2) { rs = 0; rph ^= 1; }
          break;
        }
        const int n_blocks = it.n_blocks, block0 = it.block0, shared_blocks = it.shared_blocks;
        const bool row_valid = i_seq < it.n_seq && h < it.heads;
        const int kv = row_valid ? it.kv[i_seq] : 0, shared_keys = kv > 0 ? it.shared_pages * HS_PAGE_SIZE : 0;
        // the row sees the first shared_keys of the shared blocks' keys, and lo .. hi - 1 of its half's others
        const int my_half = i_seq >= it.first_b ? 1 : 0;
        const int lo = row_valid ? (it.begin[i_seq] - (my_half ? it.pages_a : 0)) * HS_PAGE_SIZE : 0, hi = lo + kv - shared_keys;
        const float slope = MOD && a.slopes && row_valid ? a.slopes[it.head0 + h] * 1.4426950408889634f : 0.f;
        m_ref = -INFINITY;
        l_run = 0.f;
#pragma unroll 1
        for (int j = 0; j < n_blocks; ++j) {
          const uint32_t b = g + j, buf = b & 1, ph = (b >> 1) & 1;
          const int block = block0 + j;
          const bool common = block < shared_blocks;
          int in_half = block;
          const bool mine = common || it.half_of(block - shared_blocks, in_half) == my_half;
          const int key0 = in_half * SA_KEYS + half * 32;          // the thread's first key
          // bits of the keys seen, 32 and 32
          uint32_t seen[2];
#pragma unroll
          for (int c = 0; c < 2; ++c)
            seen[c] = !mine ? 0u : common ? first_bits(shared_keys - key0 - 32 * c) : first_bits(hi - key0 - 32 * c) & ~first_bits(lo - key0 - 32 * c);
          if (n_chunks == 1) seen[1] = 0;
          ok = __all_sync(0xffffffffu, mbar_wait(&tm.s_full[buf], ph, abort_flag, a.status));
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t s_col = t_lane + buf * SA_KEYS;
          if (__any_sync(0xffffffffu, (seen[0] | seen[1]) != 0)) {
            // A row sees all of a page's keys or none, but for a sequence's last page: only a warp that meets one of those masks key by key.
            auto page_seen = [&](int c, int q) { return ((c ? seen[1] : seen[0]) >> (16 * q) & 0xffffu) != 0; };
            auto in_part = [](uint32_t w) { return ((w & 0xffffu) != 0 && (w & 0xffffu) != 0xffffu) || ((w >> 16) != 0 && (w >> 16) != 0xffffu); };
            const bool partial = __any_sync(0xffffffffu, in_part(seen[0]) || in_part(seen[1]));
            auto mask = [&](int c, uint32_t to) {
              const uint32_t bits = c ? seen[1] : seen[0];
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (!(bits & (1u << k))) sreg[k] = to;
            };
            // Raw scores.  Capped ones that are not seen are NaN, which maxima and minima pass over.
            auto load = [&](int c, bool with_mask) {
              tmem_ld32(s_col + (half + c) * 32, sreg);
              tmem_ld_wait();
              if (with_mask && partial) mask(c, MOD ? 0x7fffffffu : 0xff800000u);
            };
            // The largest (or smallest) of the pages that are seen, in two chains each with three operands at a time.
            auto over_pages = [&](int c, float none, auto op) {
              float x[2];
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                auto at = [&](int k) { return __uint_as_float(sreg[16 * q + k]); };
                float y = op(at(0), at(2), at(4)), z = op(at(1), at(3), at(5));
#pragma unroll
                for (int k = 6; k < 14; k += 4) {
                  y = op(y, at(k), at(k + 2));
                  z = op(z, at(k + 1), at(k + 3));
                }
                y = op(y, at(14), at(15));
                x[q] = page_seen(c, q) ? op(y, z, z) : none;
              }
              return op(x[0], x[1], x[1]);
            };
            auto largest = [&](int c) { return over_pages(c, -INFINITY, [](float x, float y, float z) { return max3(x, y, z); }); };
            auto smallest = [&](int c) { return over_pages(c, INFINITY, [](float x, float y, float z) { return min3(x, y, z); }); };
            // While the warp's scores allow a polynomial for the cap, that of the largest score is the largest one, and the reference is part of its last
            // multiply-add.  A bias, a mask key by key, or the cap beyond, has to be worked out before the maximum is known, and once more behind it.
            float mx = -INFINITY;
            int degree = 0;
            bool direct = !MOD;
            if (!MOD || sc.out != 0.f) {
              float least = INFINITY;
#pragma unroll 1
              for (int c = n_chunks - 1; c >= 0; --c) {
                load(c, true);
                mx = fmaxf(mx, largest(c));
                if (MOD) least = fminf(least, smallest(c));
              }
              if (MOD) {
                const float u = mx > -INFINITY ? fmaxf(mx * mx, least * least) : 0.f;
                // one vote: the worst row's polynomial (6: degree three, 4: five, 0: none)
                const unsigned vote = __reduce_and_sync(0xffffffffu, u <= sc.limit3 ? 6u : u <= sc.limit5 ? 4u : 0u);
                degree = vote == 6 ? 3 : vote == 4 ? 5 : 0;
                direct = degree != 0 && a.slopes == nullptr && !partial;
                if (direct && mx > -INFINITY) {
                  const float v = mx * mx;
                  mx *= degree == 3 ? fmaf(fmaf(fmaf(sc.c3[3], v, sc.c3[2]), v, sc.c3[1]), v, sc.c3[0])
                                    : fmaf(fmaf(fmaf(fmaf(fmaf(sc.c5[5], v, sc.c5[4]), v, sc.c5[3]), v, sc.c5[2]), v, sc.c5[1]), v, sc.c5[0]);
                }
              }
            }
            auto finish = [&](int c) {                   // scores with cap and bias, in log2 units
              load(c, false);
              // the row is at position kv - 1, element e of the chunk at kv - 1 - (base - e)
              const float base = float(kv - 1 - (common ? key0 : shared_keys + key0 - lo) - 32 * c);
              const F2 base2 = f2(-slope * base, -slope * base), slope2 = f2(slope, slope), in2 = f2(sc.in, sc.in);
              auto all = [&](auto score) {               // score(pair of raw scores, what to add)
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  float y0, y1;
                  split(score(f2(__uint_as_float(sreg[e]), __uint_as_float(sreg[e + 1])), fma2(slope2, f2(float(e), float(e + 1)), base2)), y0, y1);
                  sreg[e] = __float_as_uint(y0);
                  sreg[e + 1] = __float_as_uint(y1);
                }
              };
              if (sc.out == 0.f) all([&](F2 s, F2 plus) { return fma2(s, in2, plus); });
              else if (degree == 3) all([&](F2 s, F2 plus) { return odd_poly(s, sc.c3, plus); });
              else if (degree == 5) all([&](F2 s, F2 plus) { return odd_poly(s, sc.c5, plus); });
              else {
                all([&](F2 s, F2 plus) {
                  float s0, s1;
                  split(s, s0, s1);
                  return fma2(f2(tanh_any(s0 * sc.in), tanh_any(s1 * sc.in)), f2(sc.out, sc.out), plus);
                });
              }
              if (partial) mask(c, 0xff800000u);         // -infinity
            };
            if (MOD && !direct) {
              mx = -INFINITY;
#pragma unroll 1
              for (int c = n_chunks - 1; c >= 0; --c) {
                finish(c);
                mx = fmaxf(mx, largest(c));
              }
            }
            // the reference maximum moves only when the block's maximum is far above it
            const float unit = MOD ? 1.f : sc.in;
            float alpha = 1.f;
            const bool move = mx > -INFINITY && (m_ref == -INFINITY || (mx - m_ref) * unit > kRefSlack);
            if (move) {
              alpha = m_ref == -INFINITY ? 0.f : fast_exp2((m_ref - mx) * unit);
              m_ref = mx;
            }
            const bool rescale = j > 0 && __any_sync(0xffffffffu, move);
            const float neg_ms = m_ref == -INFINITY ? 0.f : -m_ref * unit;
            const F2 neg2 = f2(neg_ms, neg_ms), unit2 = f2(unit, unit);
            float sum = 0.f;
#pragma unroll 1
            for (int c = 0; c < n_chunks; ++c) {
              if (c > 0) {
                if (MOD && !direct) finish(c);
                else load(c, true);
              }
              // log2 of the weights, a page's eight pairs step by step, so that the pairs' steps overlap; P over S: column e of row r = keys 2 e, 2 e + 1
              uint32_t pk[16];
              auto weights = [&](auto score) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                  F2 x[8], sums[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
                  for (int i = 0; i < 8; ++i) x[i] = f2(__uint_as_float(sreg[16 * q + 2 * i]), __uint_as_float(sreg[16 * q + 2 * i + 1]));
                  score(x);
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    float y0, y1;
                    split(x[i], y0, y1);
                    y0 = fast_exp2(y0);
                    y1 = fast_exp2(y1);
                    sums[i & 1] = add2(sums[i & 1], f2(y0, y1));
                    // (at most 2^kRefSlack, rounded once for the product with v in 16 bits; the sums keep fp32)
                    const uint32_t word = pack_16<F16>(y0, y1);
                    pk[8 * q + i] = page_seen(c, q) ? word : 0u;
                  }
                  float sum_a, sum_b;
                  split(add2(sums[0], sums[1]), sum_a, sum_b);
                  sum += page_seen(c, q) ? sum_a + sum_b : 0.f;
                }
              };
              auto poly = [&](F2(&x)[8], const auto& k, auto n) {
                F2 u[8], q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = mul2(x[i], x[i]);
#pragma unroll
                for (int i = 0; i < 8; ++i) q[i] = f2(k[n - 1], k[n - 1]);
#pragma unroll
                for (int d = n - 2; d >= 0; --d)
#pragma unroll
                  for (int i = 0; i < 8; ++i) q[i] = fma2(q[i], u[i], f2(k[d], k[d]));
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = fma2(q[i], x[i], neg2);
              };
              if (!MOD || !direct) {
                weights([&](F2(&x)[8]) {
#pragma unroll
                  for (int i = 0; i < 8; ++i) x[i] = fma2(x[i], unit2, neg2);
                });
              } else if (degree == 3) {
                weights([&](F2(&x)[8]) { poly(x, sc.c3, std::integral_constant<int, 4>()); });
              } else {
                weights([&](F2(&x)[8]) { poly(x, sc.c5, std::integral_constant<int, 6>()); });
              }
              tmem_st16(s_col + (half + c) * 16, pk);
            }
            l_run = l_run * alpha + sum;
            if (copies == 2) {                           // the other copy's keys
              uint32_t none[16] = {};
              tmem_st16(s_col + (half ^ 1) * 16, none);
            }
            if (rescale) {
              // O must be at rest: the P V product of the previous block has completed (the next cannot be issued before this team hands over P)
              ok = __all_sync(0xffffffffu, mbar_wait(&tm.o_full[(b - 1) & 1], ((b - 1) >> 1) & 1, abort_flag, a.status));
              if (!ok) break;
              tc_fence_after_sync();
#pragma unroll 1
              for (int c = 0; c < DH; c += 32) {
                tmem_ld32(t_lane + G_::O0 + c, sreg);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) sreg[e] = __float_as_uint(__uint_as_float(sreg[e]) * alpha);
                tmem_st32(t_lane + G_::O0 + c, sreg);
              }
            }
          } else {
            uint32_t none[16] = {};
            tmem_st16(s_col, none);
            tmem_st16(s_col + 16, none);
          }
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&tm.p_full[buf]);
        }
        if (!ok) break;
        // ------------------------------------------------------------ the item's end
        g += n_blocks;
        ok = __all_sync(0xffffffffu, mbar_wait(&tm.o_full[(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag, a.status));
        if (!ok) break;
        tc_fence_after_sync();
        middle = it.middle;
        if (!middle) {
          float f;
          const float2 total = row_total(f, ok);
          if (!ok || !deliver(it, total, f)) break;
          if (it.parts > 1) {
            __threadfence();
            __syncwarp();
            if (lane == 0) arrived(it.number, it.parts, 1);
          }
        }
        tc_fence_before_sync();
        fence_proxy_async();                             // (Q's place was written)
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&tm.q_empty);
          mbar_arrive(&tm.ring_empty[rs]);
        }
        if (++rs == 2) { rs = 0; rph ^= 1; }
      }
    }
    // -------------------------------------------------------------- the share's end
    if (tid == 0) bar->middle[turn & 1] = middle;
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (*abort_flag) break;
    if (bar->middle[turn & 1]) {
      // The tile in the middle, the last item of both teams, in the ring's slot in front of the last.  All rows of both go through their own Q, K and V, which are idle,
      // [columns / 4][128 rows]; then a thread has some columns of one row, and adds up its two or four places.
      const Item& it = tm.ring[rs];
      const int parts = it.parts, number = it.number;    // (the slot is given back: behind the last barrier here the next share's first item goes into it)
      if (warp < 8) {
        float4* dst = reinterpret_cast<float4*>(q_smem);
        tm.ml[r] = make_float2(row_reference(), l_run);
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          tmem_ld32(t_lane + G_::O0 + c, sreg);
          tmem_ld_wait();
#pragma unroll
          for (int u = 0; u < 8; ++u)
            dst[(c / 4 + u) * SA_ROWS + r] = make_float4(__uint_as_float(sreg[4 * u]), __uint_as_float(sreg[4 * u + 1]), __uint_as_float(sreg[4 * u + 2]),
                                                         __uint_as_float(sreg[4 * u + 3]));
        }
      }
      __syncthreads();
      if (warp < 8) {
        const int row_in = tid & (copy_rows - 1), i_seq = row_in / p.heads, h = row_in - i_seq * p.heads, columns = DH * copy_rows / 256, c0 = tid / copy_rows * columns;
        if (i_seq < it.n_seq && h < it.heads) {
          const float4* src[4];
          float w[4], top = -INFINITY, l = 0.f;
          float2 x[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {                  // (team q % 2, copy q / 2)
            src[q] = reinterpret_cast<const float4*>(smem + (q & 1) * G_::TEAM_BYTES) + (row_in + (q >> 1) * copy_rows) % SA_ROWS;
            x[q] = q < 2 * copies ? reinterpret_cast<const Team*>(smem + G_::TEAMS)[q & 1].ml[(row_in + (q >> 1) * copy_rows) % SA_ROWS] : make_float2(-INFINITY, 0.f);
            top = fmaxf(top, x[q].x);
          }
          const float zero = top == -INFINITY ? 0.f : top;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            w[q] = fast_exp2(x[q].x - zero);
            l = fmaf(x[q].y, w[q], l);
          }
          const bool whole = parts == 1;
          const int64_t row = it.seq0 + i_seq;
          const int head = it.head0 + h;
          RowsPart<DH>& part = reinterpret_cast<RowsPart<DH>*>(static_cast<char*>(a.workspace) + kWsScratch)[it.slot];
          uint16_t* dst = static_cast<uint16_t*>(a.o) + row * a.o_stride + head * DH;
          if (c0 == 0) {
            if (!whole) __stcg(&part.ml[row_in], make_float2(top, l));
            else if (a.lse) a.lse[row * a.n_q_heads + head] = l == 0.f ? -INFINITY : kLn2 * (top + log2f(l));
          }
          const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
          for (int q = 0; q < 4; ++q) w[q] *= inv;
          float none = 0.f;
#pragma unroll 1
          for (int c = c0; c < c0 + columns; c += 8) {
            float4 y[2] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (q >= 2 * copies) continue;
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float4 v = src[q][(c / 4 + e) * SA_ROWS];
                y[e].x = fmaf(v.x, w[q], y[e].x);
                y[e].y = fmaf(v.y, w[q], y[e].y);
                y[e].z = fmaf(v.z, w[q], y[e].z);
                y[e].w = fmaf(v.w, w[q], y[e].w);
              }
            }
            if (whole) {
              none = fmaf((y[0].x + y[0].y) + (y[0].z + y[0].w) + ((y[1].x + y[1].y) + (y[1].z + y[1].w)), 0.f, none);
              *reinterpret_cast<uint4*>(dst + c) = make_uint4(pack_16<F16>(y[0].x, y[0].y), pack_16<F16>(y[0].z, y[0].w), pack_16<F16>(y[1].x, y[1].y),
                                                              pack_16<F16>(y[1].z, y[1].w));
            } else {
              __stcg(&part.o[c / 4][row_in], y[0]);
              __stcg(&part.o[c / 4 + 1][row_in], y[1]);
            }
          }
          if (none != 0.f && l < INFINITY) bar->again = 1;
        }
        fence_proxy_async();                             // (Q's place was written)
      }
      tc_fence_before_sync();
      __syncthreads();
      tc_fence_after_sync();
      if (tid == 0 && parts > 1) {
        __threadfence();                                 // (of both teams' part, which the barrier has brought here)
        arrived(number, parts, 4);
      }
    }
  }

  // --------------------------------------------------------------- teardown --
  __syncwarp();
  if (*abort_flag) drain_after_abort();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, SA_TMEM);
  }
  const int n_joins = bar->n_joins;
  if (n_joins > 0) __threadfence();
#pragma unroll 1
  for (int i = 0; i < n_joins; ++i) {
    const int number = bar->joins[i], place = plan.place_of(number), blocks = plan.blocks_of(number), end = place + blocks + SA_ITEM_COST, f = plan.first_share(place);
    const int t_ = number / units, unit = number - t_ * units, g = find_last(plan.tile, n_groups, t_);
    const int s0 = int(plan.group[g]) + (t_ - int(plan.tile[g])) * p.tile_seqs, n = min(int(plan.group[g + 1]) - s0, p.tile_seqs);
    const int hk = unit / p.chunks, heads_all = a.n_q_heads / a.n_kv_heads, in_head = (unit - hk * p.chunks) * p.heads, heads = min(heads_all - in_head, p.heads);
    // The slots of the parts, in order, and what each row's parts weigh (Q, K and V are idle: both lie there), [part][row]; then sums of the parts.
    int* slots = reinterpret_cast<int*>(smem);
    float* weight = reinterpret_cast<float*>(smem + 1024);
    __syncthreads();
    if (warp == 0) {
      int parts = 0;
      for (int k0 = f; k0 < plan.shares && plan.share_begin(k0) < end; k0 += 32) {
        const int k = k0 + lane;
        bool has = false;
        if (k < plan.shares && plan.share_begin(k) < end) {
          const int from = k == f ? 0 : plan.cut_block(place, blocks, plan.share_begin(k));
          has = from < (plan.share_begin(k + 1) < end ? plan.cut_block(place, blocks, plan.share_begin(k + 1)) : blocks);
        }
        const unsigned who = __ballot_sync(0xffffffffu, has);
        if (has) slots[1 + parts + __popc(who & ((1u << lane) - 1u))] = 2 * k + (place < plan.share_begin(k) ? 0 : 1);
        parts += __popc(who);
      }
      if (lane == 0) slots[0] = parts;
    }
    __syncthreads();
    const int parts = slots[0], n_rows = n * p.heads;
    const RowsPart<DH>* rows_parts = reinterpret_cast<const RowsPart<DH>*>(static_cast<const char*>(a.workspace) + kWsScratch);
    for (int r = tid; r < n_rows; r += SA_THREADS) {
      const int i_seq = r / p.heads, h = r - i_seq * p.heads;
      if (h >= heads) continue;
      float top = -INFINITY, l = 0.f;
#pragma unroll 1
      for (int k0 = 0; k0 < parts; k0 += 4) {
        float2 q[4];
        float next = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = k0 + u < parts ? __ldcg(&rows_parts[slots[1 + k0 + u]].ml[r]) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          next = fmaxf(next, q[u].x);
          if (k0 + u < parts) weight[(k0 + u) * SA_ROWS + r] = q[u].x;
        }
        const float zero = next == -INFINITY ? 0.f : next;
        l *= fast_exp2(top - zero);
#pragma unroll
        for (int u = 0; u < 4; ++u) l = fmaf(fast_exp2(q[u].x - zero), q[u].y, l);
        top = next;
      }
      const float zero = top == -INFINITY ? 0.f : top, inv = l == 0.f ? 0.f : 1.f / l;
      for (int k = 0; k < parts; ++k) weight[k * SA_ROWS + r] = fast_exp2(weight[k * SA_ROWS + r] - zero) * inv;
      if (a.lse) a.lse[int64_t(s0 + i_seq) * a.n_q_heads + hk * heads_all + in_head + h] = l == 0.f ? -INFINITY : kLn2 * (top + log2f(l));
    }
    __syncthreads();
    // A thread has eight coordinates each of all its rows at once, and a part's are asked for together: it is one SM's way to the L2 that bounds it.
    constexpr int PIECES = (SA_ROWS * (DH / 8) + SA_THREADS - 1) / SA_THREADS;
    const int n_pieces = n_rows * (DH / 8);
    float4 o[PIECES][2];
    int at[PIECES];                                      // row, and the place of its coordinates in a part
#pragma unroll
    for (int y = 0; y < PIECES; ++y) {
      const int x = min(tid + y * SA_THREADS, n_pieces - 1), c = x / n_rows;
      at[y] = 2 * c * SA_ROWS + x - c * n_rows;
      o[y][0] = o[y][1] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll 1
    for (int k = 0; k < parts; ++k) {
      const RowsPart<DH>& from = rows_parts[slots[1 + k]];
      float4 v[PIECES][2];
#pragma unroll
      for (int y = 0; y < PIECES; ++y) {
        if (y * SA_THREADS >= n_pieces) continue;
        v[y][0] = __ldcg(&from.o[0][0] + at[y]);
        v[y][1] = __ldcg(&from.o[0][0] + at[y] + SA_ROWS);
      }
#pragma unroll
      for (int y = 0; y < PIECES; ++y) {
        if (y * SA_THREADS >= n_pieces) continue;
        const float w = weight[k * SA_ROWS + at[y] % SA_ROWS];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[y][e].x = fmaf(w, v[y][e].x, o[y][e].x);
          o[y][e].y = fmaf(w, v[y][e].y, o[y][e].y);
          o[y][e].z = fmaf(w, v[y][e].z, o[y][e].z);
          o[y][e].w = fmaf(w, v[y][e].w, o[y][e].w);
        }
      }
    }
#pragma unroll
    for (int y = 0; y < PIECES; ++y) {
      const int r = at[y] % SA_ROWS, c = at[y] / (2 * SA_ROWS), i_seq = r / p.heads, h = r - i_seq * p.heads;
      if (tid + y * SA_THREADS >= n_pieces || h >= heads) continue;
      if (((o[y][0].x + o[y][0].y) + (o[y][0].z + o[y][0].w) + ((o[y][1].x + o[y][1].y) + (o[y][1].z + o[y][1].w))) * 0.f != 0.f && weight[r] == weight[r]) bar->again = 1;
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.o) + int64_t(s0 + i_seq) * a.o_stride + (hk * heads_all + in_head + h) * DH + c * 8) =
          make_uint4(pack_16<F16>(o[y][0].x, o[y][0].y), pack_16<F16>(o[y][0].z, o[y][0].w), pack_16<F16>(o[y][1].x, o[y][1].y),
                     pack_16<F16>(o[y][1].z, o[y][1].w));
    }
  }

  if (n_joins > 0) __syncthreads();
  if (bar->again) finished_again<DH, F16>(p, plan, bar->joins, n_joins);
}

template <int DH>
constexpr int sa_smem() {
  return SharedGeom<DH>::SMEM > kMinSmemBytes ? SharedGeom<DH>::SMEM : kMinSmemBytes;
}

using SharedKernel = void (*)(SharedParams);
template <int DH>
SharedKernel pick(bool f16, bool mod) {
  if (f16) return mod ? shared_attention_kernel<DH, true, true> : shared_attention_kernel<DH, true, false>;
  return mod ? shared_attention_kernel<DH, false, true> : shared_attention_kernel<DH, false, false>;
}
SharedKernel pick(int dh, bool f16, bool mod) { return dh == 128 ? pick<128>(f16, mod) : pick<64>(f16, mod); }

}  // namespace

// Groups whose rows are 64 or fewer on average stand in the matrix twice.
SharedTile shared_attention_tile(const hs_shared_attention_t& a) {
  SharedTile t;
  const int heads = a.n_q_heads / a.n_kv_heads, seqs = (a.n_seqs + a.n_groups - 1) / a.n_groups;
  t.copies = int64_t(heads) * seqs <= SA_ROWS / 2 ? 2 : 1;
  t.heads = std::min(heads, SA_ROWS);
  t.seqs = SA_ROWS / t.copies / t.heads;
  return t;
}

cudaError_t shared_attention_set_attributes() {
  for (int i = 0; i < 8; ++i) {
    const int dh = i & 1 ? 128 : 64;
    const cudaError_t e = set_kernel_smem(pick(dh, i & 2, i & 4), dh == 128 ? sa_smem<128>() : sa_smem<64>());
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_shared_attention(const hs_shared_attention_t& a, const CUtensorMap& tm_q, int sm_count, int sm_budget, cudaStream_t stream) {
  SharedParams p{};
  p.tm_q = tm_q;
  p.a = a;
  p.score = score_scale(a.scale, a.cap);
  const SharedTile tile = shared_attention_tile(a);
  p.heads = tile.heads;
  p.chunks = (a.n_q_heads / a.n_kv_heads + p.heads - 1) / p.heads;
  p.tile_seqs = tile.seqs;
  p.half_seqs = (SA_ROWS / tile.copies / 2 + tile.heads - 1) / tile.heads;
  p.copies = tile.copies;
  p.shares = share_count(sm_count);
  // Without a cap and slopes the kernel masks and compares raw scores and multiplies by the scale in the exponent: right for a positive scale only.  The other
  // instantiation scales first.
  const bool modified = a.cap > 0.f || a.slopes != nullptr || !(a.scale > 0.f);
  return launch_step_kernel(pick(a.head_dim, a.type == HS_TYPE_F16, modified), std::min(sm_budget, p.shares), SA_THREADS,
                            a.head_dim == 128 ? sa_smem<128>() : sa_smem<64>(), stream, true, p);
}

}  // namespace hs
