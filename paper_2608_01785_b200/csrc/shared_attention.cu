// Attention of one new token per sequence over the paged cache, where the sequences of a group share their first keys, on the 5th-generation
// tensor cores; planned on the device.
//
//   tile      sequences of one group that follow one another, all query heads of one KV head: up to 128 rows of a matrix, sequence after sequence.
//   keys      the tile's keys are one line of blocks of 64: the group's shared pages, read once for all rows, then the pages of each sequence's own keys, one sequence
//             behind the other.  A row sees the shared keys and a run of the others; what it does not see is masked, and a warp whose 32 rows see nothing
//             of a block gives it the weight 0 and goes on.  (The products with rows that see nothing cost nothing that counts: a block's two products take 256 cycles
//             of the tensor cores, its 32 KB take 1400 to come.)
//   streams   a block of threads works on one tile at a time with two running softmaxes over the same rows, for the even and the odd blocks: S = Q K^T into tensor memory,
//             one thread per row, P back over S, O += P V.  They are added at the tile's end.
//   shares    all tiles' lines, one after the other, are cut into equal shares, about one per SM of the device, wherever the cut falls.  A tile that is cut leaves its
//             parts in the workspace; the block that delivers the last one joins them, in order.  Where the cuts lie depends on the lengths and the device,
//             never on the budget, and a block takes one share after the other.
//
// Every block plans for itself, from the lengths, in shared memory.
#include <math.h>

#include <algorithm>

#include "paged_tiles.cuh"

namespace hs {
namespace {

constexpr int SA_THREADS = 448, SA_KEYS = 64, SA_STAGES = 4, SA_ROWS = 128;
constexpr int SA_TMEM = 512;
constexpr int SA_ITEM_COST = 3;                          // blocks that take as long as a tile's beginning and end
constexpr int SA_MIN_SHARE = 6, SA_MIN_PART = 2;         // blocks, with the tiles' costs; blocks of a part
constexpr float kRefSlack = 8.f;                         // log2 units by which a row's running maximum may exceed its reference
constexpr float kLn2 = 0.6931471805599453f;

struct SharedParams {
  CUtensorMap tm_kv, tm_q;
  hs_shared_attention_t a;
  ScoreScale score;
  int heads, chunks;                                     // query heads of a tile; groups of them per KV head
  int tile_seqs;                                         // sequences of a tile
  int shares;                                            // at most
};

// A tile's part in the workspace: outputs relative to the row's reference, four coordinates of all rows after one another, then (reference in log2 units, sum).
template <int DH>
struct RowsPart {
  float4 o[DH / 4][SA_ROWS];
  float2 ml[SA_ROWS];
};

// One item -- a tile, or the part of it that a share has -- the same in every role.
struct Item {
  int valid;
  int seq0, n_seq;                                       // the tile's sequences
  int hk, head0, heads;                                  // KV head, first query head, query heads
  int table;                                             // the sequence whose block table row has the shared pages
  int shared_pages, shared_blocks;
  int block0, n_blocks;                                  // of the tile's line
  int parts, slot;                                       // parts of the tile (1: not cut), and where this one goes
  int number, unused;                                    // of the tile and its head, in the line
  int begin[SA_ROWS + 1];                                // own pages in front of each sequence's
  int kv[SA_ROWS];                                       // keys of each sequence
};
struct Barriers {
  uint64_t q_full, q_empty;
  uint64_t k_full[SA_STAGES], k_empty[SA_STAGES], v_full[SA_STAGES], v_empty[SA_STAGES];
  uint64_t s_full[2][2], p_full[2][2], o_full[2][2];
  uint64_t ring_full[2], ring_empty[2];
  uint64_t end_full, end_read;                           // an item's end: (reference, sum) of all rows are there; O has been read
  alignas(16) int v_keys[SA_STAGES][4];                              // keys of each page of a V block that some row sees, the first ones
  uint32_t tmem_base;
  int abort_flag, n_joins;
  int warp_sum[SA_THREADS / 32];
};

template <int DH>
struct SharedGeom {
  static constexpr int HALVES = DH / 64;
  static constexpr int Q_BYTES = HALVES * 16384;         // [half][128 rows][128 B]
  static constexpr int KV_BYTES = HALVES * 8192;         // K (or V) of a block: [half][4 pages][16 keys][128 B]
  static constexpr int O0 = 256;                         // tensor-memory columns: S(stream, buffer) at stream * 128 + buffer * 64, O(stream) from here on
  static constexpr int BARRIERS = Q_BYTES + 2 * SA_STAGES * KV_BYTES, ITEMS = BARRIERS + 1024, ML = ITEMS + 2 * int(sizeof(Item)),
                       JOINS = ML + 2 * SA_ROWS * 8, PLAN = JOINS + kMaxShares * 4;
  // the plan: costs of tiles (running sums), shared pages of groups; first sequences and tiles of groups in 16 bits
  static constexpr int SMEM = 1024 + PLAN + (HS_DEVICE_MAX_SEQS + 2) * (4 + 4 + 2 + 2);
};
static_assert(sizeof(Barriers) <= 1024 && sizeof(Item) % 8 == 0 && SharedGeom<128>::SMEM <= 227 * 1024, "fits one SM");
static_assert(size_t(kMaxShares) * 2 * sizeof(RowsPart<128>) <= kWsScratchBytes, "two parts per share");
static_assert(kWsSharedQueue + kMaxShares * 4 <= kWsScratch && HS_DEVICE_MAX_SEQS < 65536, "one word per share");

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
  int tiles, line, shares;
};

template <int DH, bool F16, bool MOD>
__global__ void __launch_bounds__(SA_THREADS, 1) shared_attention_kernel(const __grid_constant__ SharedParams p) {
  using G_ = SharedGeom<DH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_smem = smem;
  uint8_t* k_smem = q_smem + G_::Q_BYTES;
  uint8_t* v_smem = k_smem + SA_STAGES * G_::KV_BYTES;
  Barriers* bar = reinterpret_cast<Barriers*>(smem + G_::BARRIERS);
  Item* ring = reinterpret_cast<Item*>(smem + G_::ITEMS);
  float2(*ml)[SA_ROWS] = reinterpret_cast<float2(*)[SA_ROWS]>(smem + G_::ML);            // [stream][row]
  int* joins = reinterpret_cast<int*>(smem + G_::JOINS);                                 // tiles that this block joins
  volatile int* abort_flag = &bar->abort_flag;
  const hs_shared_attention_t& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = int(threadIdx.x);
  const int n_seqs = a.n_seqs, n_groups = a.n_groups, units = a.n_kv_heads * p.chunks;
  const int most_keys = row_tokens(a.max_pages_per_seq);

  if (tid == 0) {
    mbar_init(&bar->q_full, 1);
    mbar_init(&bar->q_empty, 2);                         // one arrival per MMA thread
    for (int i = 0; i < SA_STAGES; ++i) {
      mbar_init(&bar->k_full[i], 2);
      mbar_init(&bar->k_empty[i], 1);
      mbar_init(&bar->v_full[i], 2);
      mbar_init(&bar->v_empty[i], 1);
    }
    for (int t = 0; t < 2; ++t)
      for (int i = 0; i < 2; ++i) {
        mbar_init(&bar->s_full[t][i], 1);
        mbar_init(&bar->p_full[t][i], 128);
        mbar_init(&bar->o_full[t][i], 1);
      }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar->ring_full[i], 1);
      mbar_init(&bar->ring_empty[i], 13);                // eight softmax warps, two MMA warps, three further producers
    }
    mbar_init(&bar->end_full, 256);
    mbar_init(&bar->end_read, 256);
    bar->abort_flag = 0;
    bar->n_joins = 0;
    fence_barrier_init();
    tma_prefetch_desc(&p.tm_kv);
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
    int* shared = cost + HS_DEVICE_MAX_SEQS + 2;
    uint16_t* group = reinterpret_cast<uint16_t*>(shared + HS_DEVICE_MAX_SEQS + 2);
    uint16_t* tile = group + HS_DEVICE_MAX_SEQS + 2;
    int wrong = 0;
    for (int g = tid; g <= n_groups; g += SA_THREADS) {
      const int b = a.group_begin[g];
      wrong |= b < 0 || b > n_seqs || (g < n_groups && (a.group_begin[g + 1] < b || a.shared_len[g] < 0));
      group[g] = uint16_t(b);
      shared[g] = 0x7fffffff;                            // (the fewest keys of a sequence that has some)
    }
    wrong = __syncthreads_or(wrong);
    if (wrong) {
      if (tid == 0 && blockIdx.x == 0) atomicExch(a.status, kErrInvalidArg);
      if (warp == 9) tmem_dealloc(tmem, SA_TMEM);
      return;
    }
    plan.tiles = running_sums(n_groups, bar->warp_sum, [&](int g) { return (int(group[g + 1]) - int(group[g]) + p.tile_seqs - 1) / p.tile_seqs; },
                              [&](int g, int sum) { tile[g] = uint16_t(sum); });
    if (tid == 0) tile[n_groups] = uint16_t(plan.tiles);
    const int s_end = group[n_groups];
    for (int s = int(group[0]) + tid; s < s_end; s += SA_THREADS) {
      const int kv = a.kv_len[s];
      if ((kv < 0 || kv > most_keys) && blockIdx.x == 0) atomicExch(a.status, kErrBadBlockTable);
      const int keys = keys_of(s);
      if (keys > 0) atomicMin(&shared[find_last(group, n_groups, s)], keys);
    }
    for (int t = tid; t < plan.tiles; t += SA_THREADS) cost[t] = 0;
    __syncthreads();
    for (int g = tid; g < n_groups; g += SA_THREADS) shared[g] = shared[g] == 0x7fffffff ? 0 : min(shared[g], a.shared_len[g]) / HS_PAGE_SIZE;
    __syncthreads();
    for (int s = int(group[0]) + tid; s < s_end; s += SA_THREADS) {
      const int g = find_last(group, n_groups, s), keys = keys_of(s);
      if (keys > 0) atomicAdd(&cost[tile[g] + (s - group[g]) / p.tile_seqs], (keys + HS_PAGE_SIZE - 1) / HS_PAGE_SIZE - shared[g]);
    }
    __syncthreads();
    // (at least one block, so that rows that see no key take the same way)
    for (int t = tid; t < plan.tiles; t += SA_THREADS) cost[t] = max((shared[find_last(tile, n_groups, t)] + 3) / 4 + (cost[t] + 3) / 4, 1) + SA_ITEM_COST;
    __syncthreads();
    const int all = running_sums(plan.tiles, bar->warp_sum, [&](int t) { return cost[t]; }, [&](int t, int sum) { cost[t] = sum; });
    if (tid == 0) cost[plan.tiles] = all;
    __syncthreads();
    plan.cost = cost;
    plan.shared = shared;
    plan.group = group;
    plan.tile = tile;
    plan.line = all * units;
    plan.shares = max(1, min(p.shares, plan.line / SA_MIN_SHARE));
  }
  // An item's number is tile * units + unit; its place in the line is the sum of the costs in front of it.
  auto cost_of = [&](int number) { return plan.cost[number / units + 1] - plan.cost[number / units]; };
  auto place_of = [&](int number) {
    const int t = number / units;
    return plan.cost[t] * units + (number - t * units) * (plan.cost[t + 1] - plan.cost[t]);
  };
  auto share_begin = [&](int k) { return int(int64_t(plan.line) * k / plan.shares); };
  auto number_at = [&](int x) {                          // of the item that has place x
    if (x >= plan.line) return plan.tiles * units;
    const int t = find_last(plan.cost, plan.tiles, x / units);
    return t * units + (x - plan.cost[t] * units) / (plan.cost[t + 1] - plan.cost[t]);
  };
  // The block of an item in front of which the cut at place x falls; not so near an end that a part would be too short.
  auto cut_block = [&](int number, int x) {
    if (number >= plan.tiles * units) return 0;
    const int blocks = cost_of(number) - SA_ITEM_COST, b = x - place_of(number) - SA_ITEM_COST;
    return b < SA_MIN_PART ? 0 : b > blocks - SA_MIN_PART ? blocks : b;
  };
  auto first_share = [&](int number) {                   // that has a place of the item
    const int x = place_of(number);
    int k = int(int64_t(x) * plan.shares / plan.line);
    while (k + 1 < plan.shares && share_begin(k + 1) <= x) ++k;
    while (share_begin(k) > x) --k;
    return k;
  };

  int rs = 0;
  uint32_t rph = 0;                                      // item ring slot / phase
  uint32_t items_seen = 0;
  uint32_t blk_base = 0;                                 // blocks of all earlier items of this thread block (K / V ring position)

  if (warp == 8 || warp >= 11) {
    // ========================================================== TMA producers ==
    // Producer 0 (warp 8) finds the items and loads pages 0, 1 of every K block; producer 1 pages 2, 3 of K; producers 2 and 3 the same of V.  Producer 0
    // loads the Q tile.  Lane l holds the id of page l % 4 of the current eight blocks' l / 4.
    const int pi = warp == 8 ? 0 : warp - 10;
    const int kv = pi >> 1, w0 = (pi & 1) * 2;
    int share = plan.tiles > 0 ? int(blockIdx.x) : plan.shares, number = -1, last = -1;           // the lead's: the share, its next item, its last one
    for (;;) {
      bool ok = true;
      if (pi == 0) {
        if (lane == 0) ok = mbar_wait(&bar->ring_empty[rs], rph ^ 1, abort_flag, a.status);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        Item& it = ring[rs];
        // the next item that has blocks
        int b0 = 0, b1 = 0;
        for (;;) {
          if (number < 0) {
            if (share >= plan.shares) break;
            number = number_at(share_begin(share));
            last = number_at(share_begin(share + 1) - 1);
          }
          const int x0 = share_begin(share), x1 = share_begin(share + 1), place = place_of(number), cost = cost_of(number);
          b0 = place < x0 ? cut_block(number, x0) : 0;
          b1 = place + cost > x1 ? cut_block(number, x1) : cost - SA_ITEM_COST;
          if (b0 < b1) break;
          if (number == last) {
            number = -1;
            share += int(gridDim.x);
          } else {
            ++number;
          }
        }
        if (number < 0) {
          if (lane == 0) it.valid = 0;
        } else {
          const int t = number / units, unit = number - t * units, g = find_last(plan.tile, n_groups, t);
          const int s0 = int(plan.group[g]) + (t - int(plan.tile[g])) * p.tile_seqs, n = min(int(plan.group[g + 1]) - s0, p.tile_seqs);
          const int shared_pages = plan.shared[g];
          int table = int(plan.group[g]);
          if (shared_pages > 0) {
            for (int s = table + lane;; s += 32) {       // (one of the group's has keys)
              const unsigned some = __ballot_sync(0xffffffffu, s < int(plan.group[g + 1]) && keys_of(s) > 0);
              if (some) {
                table = s - lane + __ffs(some) - 1;
                break;
              }
              if (s - lane >= int(plan.group[g + 1])) break;
            }
          }
          int sum = 0;
          for (int i = 0; i < n; i += 32) {
            const int keys = i + lane < n ? keys_of(s0 + i + lane) : 0;
            const int pages = keys > 0 ? (keys + HS_PAGE_SIZE - 1) / HS_PAGE_SIZE - shared_pages : 0;
            int inc = pages;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
              const int x = __shfl_up_sync(0xffffffffu, inc, o);
              if (lane >= o) inc += x;
            }
            if (i + lane < n) {
              it.begin[i + lane] = sum + inc - pages;
              it.kv[i + lane] = keys;
            }
            sum += __shfl_sync(0xffffffffu, inc, 31);
          }
          // the shares that have parts of the item
          const int place = place_of(number), end = place + cost_of(number), f = first_share(number);
          int parts = 0;
          for (int k0 = f; share_begin(k0) < end; k0 += 32) {
            const int k = k0 + lane;
            bool has = false;
            if (k < plan.shares && share_begin(k) < end) {
              const int from = k == f ? 0 : cut_block(number, share_begin(k));
              const int to = share_begin(k + 1) < end ? cut_block(number, share_begin(k + 1)) : cost_of(number) - SA_ITEM_COST;
              has = from < to;
            }
            parts += __popc(__ballot_sync(0xffffffffu, has));
            if (k0 + 32 >= plan.shares) break;
          }
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
            it.slot = 2 * share + (place < share_begin(share) ? 0 : 1);
            it.number = number;
            it.begin[n] = sum;
          }
          if (number == last) {
            number = -1;
            share += int(gridDim.x);
          } else {
            ++number;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->ring_full[rs]);
      } else {
        ok = mbar_wait(&bar->ring_full[rs], rph, abort_flag, a.status);
        if (!__all_sync(0xffffffffu, ok)) break;
      }
      const Item& it = ring[rs];
      // (a copy of what is needed: the slot is released at once, and the lead's own stays until the other roles have released it)
      const int valid = it.valid;
      if (!valid) break;
      const int n_seq = it.n_seq, hk = it.hk, shared_pages = it.shared_pages, shared_blocks = it.shared_blocks, block0 = it.block0, n_blocks = it.n_blocks;
      // Page l % 4 of block j0 + l / 4 of the item: its id, -1 where there is none, and how many of its keys are seen.
      int pages_keys = 0;
      auto page_id = [&](int j0) {
        const int j = j0 + (lane >> 2);
        pages_keys = 0;
        if (j >= n_blocks) return -1;
        int u = (block0 + j) * 4 + (lane & 3), id, keys = HS_PAGE_SIZE;
        if (block0 + j < shared_blocks) {
          if (u >= shared_pages) return -1;
          id = a.block_tables[int64_t(it.table) * a.max_pages_per_seq + u];
        } else {
          u -= shared_blocks * 4;
          if (u >= it.begin[n_seq]) return -1;
          const int i = find_last(it.begin, n_seq, u), page = shared_pages + u - it.begin[i];
          id = a.block_tables[int64_t(it.seq0 + i) * a.max_pages_per_seq + page];
          keys = min(it.kv[i] - page * HS_PAGE_SIZE, HS_PAGE_SIZE);
        }
        if (id >= 0 && id < a.num_pages) {
          pages_keys = keys;
          return id;
        }
        atomicExch(a.status, kErrBadBlockTable);
        return -1;
      };
      int pg_next = page_id(0), keys_next = pages_keys, pg_cur = -1, keys_cur = 0;
      if (pi == 0) {
        if (lane == 0) {
          ok = mbar_wait(&bar->q_empty, (items_seen & 1) ^ 1, abort_flag, a.status);
          if (ok) {
            mbar_expect_tx(&bar->q_full, G_::HALVES * p.heads * p.tile_seqs * 128);
            for (int h = 0; h < G_::HALVES; ++h)
              asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                               smem_u32(q_smem + h * 16384)),
                           "l"(reinterpret_cast<uint64_t>(&p.tm_q)), "r"(smem_u32(&bar->q_full)), "r"(h * 64), "r"(it.head0), "r"(it.seq0)
                           : "memory");
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
      }
      ++items_seen;
      for (int kb = 0; kb < n_blocks && ok; ++kb) {
        if ((kb & 7) == 0) {
          pg_cur = pg_next;
          keys_cur = keys_next;
          pg_next = page_id(kb + 8);
          keys_next = pages_keys;
        }
        const uint32_t gb = blk_base + kb;
        const uint32_t st = gb % SA_STAGES, ph = (gb / SA_STAGES) & 1;
        uint64_t* full = kv ? &bar->v_full[st] : &bar->k_full[st];
        uint8_t* dst = (kv ? v_smem : k_smem) + st * G_::KV_BYTES;
        const int l0 = (kb & 7) * 4 + w0;
        const int id0 = __shfl_sync(0xffffffffu, pg_cur, l0), id1 = __shfl_sync(0xffffffffu, pg_cur, l0 + 1);
        const int keys0 = __shfl_sync(0xffffffffu, keys_cur, l0), keys1 = __shfl_sync(0xffffffffu, keys_cur, l0 + 1);
        if (lane == 0) {
          ok = mbar_wait(kv ? &bar->v_empty[st] : &bar->k_empty[st], ph ^ 1, abort_flag, a.status);
          if (ok) {
            if (kv) {
              bar->v_keys[st][w0] = keys0;
              bar->v_keys[st][w0 + 1] = keys1;
            }
            const int mine = (id0 >= 0) + (id1 >= 0);
            if (mine > 0) mbar_expect_tx(full, mine * G_::HALVES * 2048);
            else mbar_arrive(full);                      // nothing to fetch, but the block counts on two arrivals
            for (int w = 0; w < 2; ++w) {
              const int id = w ? id1 : id0;
              if (id < 0) continue;
              const int row = (((a.layer * 2 + kv) * a.num_pages + id) * a.n_kv_heads + hk) * 16;
              for (int h = 0; h < G_::HALVES; ++h) tma_load_2d(dst + h * 8192 + (w0 + w) * 2048, &p.tm_kv, full, h * 64, row);
            }
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
      }
      __syncwarp();
      if (pi != 0 && lane == 0) mbar_arrive(&bar->ring_empty[rs]);
      if (++rs == 2) { rs = 0; rph ^= 1; }
      if (!ok) break;
      blk_base += n_blocks;
    }
  } else if (warp == 9 || warp == 10) {
    // ============================================================ MMA issuers ==
    // One issuing thread per stream (warp 9: even blocks of an item, warp 10: odd ones).
    if (lane == 0) {
      const int t = warp - 9;
      constexpr uint32_t idesc_s = idesc_16<F16>(128, SA_KEYS);
      constexpr uint32_t idesc_pv = idesc_16<F16>(128, DH) | (1u << 16);   // B (= V) is MN-major
      const uint64_t q_desc = umma_desc_kmajor_sw128(smem_u32(q_smem));
      const uint64_t k_desc0 = umma_desc_kmajor_sw128(smem_u32(k_smem));
      const uint64_t v_desc0 = umma_desc_mnmajor_sw128(smem_u32(v_smem), 8192, 1024);
      const uint32_t d_o = tmem + G_::O0 + t * DH, s_base = tmem + t * 128;
      uint32_t g_s = 0, g_pv = 0;                        // blocks of this stream whose S / whose P V has been issued, over all items
      bool ok = true;
      auto pv_block = [&](int j) -> bool {               // block j of the item
        const uint32_t gb = blk_base + j, vst = gb % SA_STAGES;
        if (!mbar_wait(&bar->v_full[vst], (gb / SA_STAGES) & 1, abort_flag, a.status)) return false;
        const uint32_t buf = g_pv & 1, bph = (g_pv >> 1) & 1;
        if (!mbar_wait(&bar->p_full[t][buf], bph, abort_flag, a.status)) return false;
        tc_fence_after_sync();
        const uint64_t vdesc = v_desc0 + uint64_t(vst * (G_::KV_BYTES >> 4));
        const uint32_t a_p = s_base + buf * SA_KEYS, acc0 = j < 2 ? 0u : 1u;     // the stream's first block overwrites O
#pragma unroll
        for (int pg = 0; pg < 4; ++pg)                   // 16 keys (one page) per MMA: 8 columns of P
          umma_ts(d_o, a_p + 8 * pg, vdesc + uint64_t(pg * (2048 >> 4)), idesc_pv, pg != 0 ? 1u : acc0);
        umma_commit(&bar->o_full[t][buf]);
        umma_commit(&bar->v_empty[vst]);
        ++g_pv;
        return true;
      };
      for (;;) {
        if (!mbar_wait(&bar->ring_full[rs], rph, abort_flag, a.status)) break;
        const int valid = ring[rs].valid, n_blocks = ring[rs].n_blocks;
        mbar_arrive(&bar->ring_empty[rs]);
        if (++rs == 2) { rs = 0; rph ^= 1; }
        if (!valid) break;
        if (!mbar_wait(&bar->q_full, items_seen & 1, abort_flag, a.status)) break;
        ++items_seen;
        if (t >= n_blocks) mbar_arrive(&bar->q_empty);
        for (int j = t; j < n_blocks && ok; j += 2) {
          const uint32_t gb = blk_base + j, kst = gb % SA_STAGES;
          if (!mbar_wait(&bar->k_full[kst], (gb / SA_STAGES) & 1, abort_flag, a.status)) { ok = false; break; }
          tc_fence_after_sync();
          const uint32_t buf = g_s & 1;
          const uint64_t kdesc = k_desc0 + uint64_t(kst * (G_::KV_BYTES >> 4));
#pragma unroll
          for (int ks = 0; ks < DH / 16; ++ks)
            umma_bf16(s_base + buf * SA_KEYS, q_desc + uint64_t((ks >> 2) * (16384 >> 4) + 2 * (ks & 3)),
                      kdesc + uint64_t((ks >> 2) * (8192 >> 4) + 2 * (ks & 3)), idesc_s, ks != 0);
          umma_commit(&bar->s_full[t][buf]);
          umma_commit(&bar->k_empty[kst]);               // the K slot, once these scores are computed
          if (j + 2 >= n_blocks) umma_commit(&bar->q_empty);       // and the Q tile after the stream's last scores
          ++g_s;
          if (j >= 2) ok = pv_block(j - 2);              // overlaps the softmax of block j
        }
        if (ok && t < n_blocks) ok = pv_block((n_blocks - 1 - t) / 2 * 2 + t);
        if (!ok) break;
        blk_base += n_blocks;
      }
    }
  } else {
    // ================================================================ softmax ==
    const int t = warp >> 2;                             // stream of this warp group
    const int r = tid & 127;                             // row of the tile = TMEM lane
    const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
    const uint32_t s_col = t * 128, o_col = G_::O0 + t * DH;
    const ScoreScale& sc = p.score;
    uint32_t g = 0;                                      // blocks this stream has processed, over all items
    for (;;) {
      bool ok = mbar_wait(&bar->ring_full[rs], rph, abort_flag, a.status);
      if (!__all_sync(0xffffffffu, ok)) break;
      const Item& it = ring[rs];
      if (!it.valid) break;
      const int n_blocks = it.n_blocks, block0 = it.block0, shared_blocks = it.shared_blocks, heads = it.heads, parts = it.parts, slot = it.slot, number = it.number;
      const int i_seq = r / p.heads, h = r - i_seq * p.heads;        // (rows of a box have room for p.heads each)
      const bool row_valid = i_seq < it.n_seq && h < heads;
      const int kv = row_valid ? it.kv[i_seq] : 0, shared_keys = kv > 0 ? it.shared_pages * HS_PAGE_SIZE : 0;
      // the row sees the first shared_keys of the shared blocks' keys, and lo .. hi - 1 of the others'
      const int lo = row_valid ? it.begin[i_seq] * HS_PAGE_SIZE : 0, hi = lo + kv - shared_keys;
      const int head = it.head0 + h;
      const int64_t row = it.seq0 + i_seq;
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->ring_empty[rs]);
      if (++rs == 2) { rs = 0; rph ^= 1; }
      const bool warp_valid = __any_sync(0xffffffffu, row_valid);
      const float slope = MOD && a.slopes && row_valid ? a.slopes[head] * 1.4426950408889634f : 0.f;

      float m_ref = -INFINITY, l_run = 0.f;              // (MOD: in log2 units; else of the raw scores, whose scale is positive)
      uint32_t sreg[32], sreg2[32];
      for (int j = t; j < n_blocks; j += 2, ++g) {
        const uint32_t buf = g & 1, bph = (g >> 1) & 1;
        const int block = block0 + j;
        const bool common = block < shared_blocks;
        const int key0 = (common ? block : block - shared_blocks) * SA_KEYS;
        uint32_t seen1, seen2;                           // bit e: key key0 + e, key0 + 32 + e
        if (common) {
          seen1 = first_bits(shared_keys - key0);
          seen2 = first_bits(shared_keys - 32 - key0);
        } else {
          seen1 = first_bits(hi - key0) & ~first_bits(lo - key0);
          seen2 = first_bits(hi - 32 - key0) & ~first_bits(lo - 32 - key0);
        }
        ok = mbar_wait(&bar->s_full[t][buf], bph, abort_flag, a.status);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after_sync();
        uint32_t pk[32];
        if (__any_sync(0xffffffffu, (seen1 | seen2) != 0)) {
          tmem_ld32(tmem + lane_base + s_col + buf * SA_KEYS, sreg);
          tmem_ld32(tmem + lane_base + s_col + buf * SA_KEYS + 32, sreg2);
          tmem_ld_wait();
          const bool masked = (seen1 & seen2) != 0xffffffffu;
          auto mask = [&](uint32_t to) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              if (!(seen1 & (1u << e))) sreg[e] = to;
              if (!(seen2 & (1u << e))) sreg2[e] = to;
            }
          };
          auto largest = [&]() {                         // four chains
            float mx[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) mx[e] = fmaxf(__uint_as_float(sreg[e]), __uint_as_float(sreg2[e]));
#pragma unroll
            for (int e = 4; e < 32; ++e) mx[e & 3] = fmaxf(mx[e & 3], fmaxf(__uint_as_float(sreg[e]), __uint_as_float(sreg2[e])));
            return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          };
          auto smallest = [&]() {
            float mn[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) mn[e] = fminf(__uint_as_float(sreg[e]), __uint_as_float(sreg2[e]));
#pragma unroll
            for (int e = 4; e < 32; ++e) mn[e & 3] = fminf(mn[e & 3], fminf(__uint_as_float(sreg[e]), __uint_as_float(sreg2[e])));
            return fminf(fminf(mn[0], mn[1]), fminf(mn[2], mn[3]));
          };
          if (MOD) {
            int degree = 0;
            if (sc.out != 0.f) {
              if (masked) mask(0u);                      // (what is not seen must not decide which polynomial the others take)
              const float top = largest(), low = smallest(), u = fmaxf(top * top, low * low);
              // one vote: the worst row's polynomial (6: degree three, 4: five, 0: none)
              const unsigned vote = __reduce_and_sync(0xffffffffu, u <= sc.limit3 ? 6u : u <= sc.limit5 ? 4u : 0u);
              degree = vote == 6 ? 3 : vote == 4 ? 5 : 0;
            }
            // the row is at position kv - 1, key e of the block at p - (base - e)
            const float base = float(kv - 1 - (common ? key0 : shared_keys + key0 - lo));
            const F2 base2 = f2(-slope * base, -slope * base), slope2 = f2(slope, slope), in2 = f2(sc.in, sc.in);
            auto finish = [&](auto score) {              // score(pair of raw scores, what to add)
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                float x0, x1;
                const F2 p1 = fma2(slope2, f2(float(e), float(e + 1)), base2), p2 = fma2(slope2, f2(float(e + 32), float(e + 33)), base2);
                split(score(f2(__uint_as_float(sreg[e]), __uint_as_float(sreg[e + 1])), p1), x0, x1);
                sreg[e] = __float_as_uint(x0);
                sreg[e + 1] = __float_as_uint(x1);
                split(score(f2(__uint_as_float(sreg2[e]), __uint_as_float(sreg2[e + 1])), p2), x0, x1);
                sreg2[e] = __float_as_uint(x0);
                sreg2[e + 1] = __float_as_uint(x1);
              }
            };
            if (degree == 3) finish([&](F2 s, F2 plus) { return odd_poly(s, sc.c3, plus); });
            else if (degree == 5) finish([&](F2 s, F2 plus) { return odd_poly(s, sc.c5, plus); });
            else if (sc.out == 0.f) finish([&](F2 s, F2 plus) { return fma2(s, in2, plus); });
            else {
              finish([&](F2 s, F2 plus) {
                float s0, s1;
                split(s, s0, s1);
                return fma2(f2(tanh_any(s0 * sc.in), tanh_any(s1 * sc.in)), f2(sc.out, sc.out), plus);
              });
            }
          }
          if (masked) mask(0xff800000u);                 // -infinity
          const float mx = largest();
          // the reference maximum moves only when the block's maximum is far above it
          const float unit = MOD ? 1.f : sc.in;
          float alpha = 1.f;
          const bool move = mx > -INFINITY && (m_ref == -INFINITY || (mx - m_ref) * unit > kRefSlack);
          if (move) {
            alpha = m_ref == -INFINITY ? 0.f : fast_exp2((m_ref - mx) * unit);
            m_ref = mx;
          }
          const bool rescale = j >= 2 && __any_sync(0xffffffffu, move);
          const float neg_ms = m_ref == -INFINITY ? 0.f : -m_ref * unit;
          const F2 neg2 = f2(neg_ms, neg_ms), unit2 = f2(unit, unit);
          F2 sums[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
          auto weights = [&](auto score) {               // score(pair of raw or finished scores) = log2 of their weights
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              float x0, x1, y0, y1;
              split(score(f2(__uint_as_float(sreg[e]), __uint_as_float(sreg[e + 1]))), x0, x1);
              split(score(f2(__uint_as_float(sreg2[e]), __uint_as_float(sreg2[e + 1]))), y0, y1);
              x0 = fast_exp2(x0);
              x1 = fast_exp2(x1);
              y0 = fast_exp2(y0);
              y1 = fast_exp2(y1);
              sums[0] = add2(sums[0], f2(x0, x1));
              sums[1] = add2(sums[1], f2(y0, y1));
              // (at most 2^kRefSlack, rounded once for the product with v in 16 bits; the sums keep fp32)
              pk[e >> 1] = pack_16<F16>(x0, x1);
              pk[16 + (e >> 1)] = pack_16<F16>(y0, y1);
            }
          };
          if (!MOD) weights([&](F2 s) { return fma2(s, unit2, neg2); });
          else weights([&](F2 s) { return add2(s, neg2); });
          float sum_a, sum_b;
          split(add2(sums[0], sums[1]), sum_a, sum_b);
          l_run = l_run * alpha + (sum_a + sum_b);
          if (rescale) {
            // O must be at rest: the stream's P V product of its previous block has completed (the next cannot be issued
            // before this warp group hands over P)
            ok = mbar_wait(&bar->o_full[t][(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag, a.status);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            tc_fence_after_sync();
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) {
              tmem_ld32(tmem + lane_base + o_col + c * 32, sreg);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) sreg[e] = __float_as_uint(__uint_as_float(sreg[e]) * alpha);
              tmem_st32(tmem + lane_base + o_col + c * 32, sreg);
            }
            tmem_st_wait();
          }
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) pk[e] = 0;
        }
        // P over the first 32 columns of the S buffer just read: column c of row r = keys 2 c, 2 c + 1
        tmem_st32(tmem + lane_base + s_col + buf * SA_KEYS, pk);
        // V rows of keys that no row sees may hold anything and must not meet the weight 0
        {
          const uint32_t gb = blk_base + j, s = gb % SA_STAGES;
          const bool w = mbar_wait(&bar->v_full[s], (gb / SA_STAGES) & 1, abort_flag, a.status);
          if (!__all_sync(0xffffffffu, w)) { ok = false; break; }
          const int4 keys = *reinterpret_cast<const int4*>(bar->v_keys[s]);
          if ((keys.x & keys.y & keys.z & keys.w) != HS_PAGE_SIZE) {
            uint8_t* vst = v_smem + s * G_::KV_BYTES;
            for (int idx = r; idx < SA_KEYS * G_::HALVES * 8; idx += 128) {
              const int u = idx & 7, half = (idx >> 3) % G_::HALVES, k = (idx >> 3) / G_::HALVES, page = k >> 4;
              if ((k & 15) < (page == 0 ? keys.x : page == 1 ? keys.y : page == 2 ? keys.z : keys.w)) continue;
              *reinterpret_cast<uint4*>(vst + half * 8192 + page * 2048 + (k & 15) * 128 + (u << 4)) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
          }
        }
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(&bar->p_full[t][buf]);
      }
      if (!ok) break;
      // -------------------------------------------------------------- the item's end
      // Both streams' last products, their (reference, sum) by row; then each half of the warps has half of the coordinates.
      if (t < n_blocks) {
        ok = mbar_wait(&bar->o_full[t][(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag, a.status);
        if (!__all_sync(0xffffffffu, ok)) break;
      }
      const float m_log2 = m_ref == -INFINITY ? -INFINITY : MOD ? m_ref : __fmul_rn(m_ref, sc.in);
      ml[t][r] = make_float2(m_log2, l_run);
      tc_fence_before_sync();
      mbar_arrive(&bar->end_full);
      ok = mbar_wait(&bar->end_full, items_seen & 1, abort_flag, a.status);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after_sync();
      const float2 other = ml[t ^ 1][r];
      const float top = fmaxf(m_log2, other.x), zero = top == -INFINITY ? 0.f : top;
      const float f_mine = fast_exp2(m_log2 - zero), f_other = fast_exp2(other.x - zero);      // (0 for a stream in which the row has seen nothing)
      const float l = t == 0 ? fmaf(l_run, f_mine, other.y * f_other) : fmaf(other.y, f_other, l_run * f_mine);
      const float f0 = t == 0 ? f_mine : f_other, f1 = n_blocks > 1 ? (t == 0 ? f_other : f_mine) : 0.f;
      if (warp_valid) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint16_t* dst = static_cast<uint16_t*>(a.o) + row * a.o_stride + head * DH;
        RowsPart<DH>& part = reinterpret_cast<RowsPart<DH>*>(static_cast<char*>(a.workspace) + kWsScratch)[slot];
#pragma unroll
        for (int c = 0; c < DH / 64; ++c) {
          const int col = t * (DH / 2) + c * 32;
          tmem_ld32(tmem + lane_base + G_::O0 + col, sreg);
          tmem_ld32(tmem + lane_base + G_::O0 + DH + col, sreg2);
          tmem_ld_wait();
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            x[e] = __uint_as_float(sreg[e]) * f0;
            if (n_blocks > 1) x[e] = fmaf(__uint_as_float(sreg2[e]), f1, x[e]);         // (else the odd stream's O is not this item's)
          }
          if (row_valid) {
            if (parts == 1) {
              uint32_t w[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) w[e] = pack_16<F16>(x[2 * e] * inv, x[2 * e + 1] * inv);
#pragma unroll
              for (int u = 0; u < 4; ++u) *reinterpret_cast<uint4*>(dst + col + u * 8) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
            } else {
#pragma unroll
              for (int u = 0; u < 8; ++u) __stcg(&part.o[col / 4 + u][r], make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]));
            }
          }
        }
        if (row_valid && t == 0) {
          if (parts > 1) __stcg(&part.ml[r], make_float2(top, l));
          else if (a.lse) a.lse[row * a.n_q_heads + head] = l == 0.f ? -INFINITY : kLn2 * (top + log2f(l));
        }
      }
      if (parts > 1) __threadfence();
      tc_fence_before_sync();
      mbar_arrive(&bar->end_read);
      ok = mbar_wait(&bar->end_read, items_seen & 1, abort_flag, a.status);
      if (!__all_sync(0xffffffffu, ok)) break;
      ++items_seen;
      if (parts > 1 && tid == 0) {
        __threadfence();
        int* done = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsSharedQueue) + first_share(number);
        if (atomicAdd(done, 1) == parts - 1) {
          *done = 0;                                     // ready for the next call
          joins[bar->n_joins++] = number;
        }
      }
      blk_base += n_blocks;
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
  if (n_joins == 0) return;
  __threadfence();
#pragma unroll 1
  for (int i = 0; i < n_joins; ++i) {
    const int number = joins[i], place = place_of(number), end = place + cost_of(number), f = first_share(number);
    const int t_ = number / units, unit = number - t_ * units, g = find_last(plan.tile, n_groups, t_);
    const int s0 = int(plan.group[g]) + (t_ - int(plan.tile[g])) * p.tile_seqs, n = min(int(plan.group[g + 1]) - s0, p.tile_seqs);
    const int hk = unit / p.chunks, heads_all = a.n_q_heads / a.n_kv_heads, in_head = (unit - hk * p.chunks) * p.heads, heads = min(heads_all - in_head, p.heads);
    // the slots of the parts, in order (ring and K / V tiles are idle: the list goes there)
    int* slots = reinterpret_cast<int*>(smem);
    __syncthreads();
    if (tid == 0) {
      int parts = 0;
      for (int k = f; k < plan.shares && share_begin(k) < end; ++k) {
        const int from = k == f ? 0 : cut_block(number, share_begin(k));
        const int to = share_begin(k + 1) < end ? cut_block(number, share_begin(k + 1)) : cost_of(number) - SA_ITEM_COST;
        if (from < to) slots[1 + parts++] = 2 * k + (place < share_begin(k) ? 0 : 1);
      }
      slots[0] = parts;
    }
    __syncthreads();
    const int parts = slots[0], n_rows = n * p.heads;
    const RowsPart<DH>* rows_parts = reinterpret_cast<const RowsPart<DH>*>(static_cast<const char*>(a.workspace) + kWsScratch);
    // a thread has a row and eight of its coordinates at a time; eight parts are on their way at a time
#pragma unroll 1
    for (int x = tid; x < n_rows * (DH / 8); x += SA_THREADS) {
      const int c = x / n_rows, r = x - c * n_rows, i_seq = r / p.heads, h = r - i_seq * p.heads;
      if (h >= heads) continue;
      float top = -INFINITY, l = 0.f;
      float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
      for (int k0 = 0; k0 < parts; k0 += 4) {
        float2 q[4];
        float4 v[2][4];
        float next = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bool there = k0 + u < parts;
          const RowsPart<DH>& from = rows_parts[slots[1 + min(k0 + u, parts - 1)]];
          q[u] = there ? __ldcg(&from.ml[r]) : make_float2(-INFINITY, 0.f);
#pragma unroll
          for (int e = 0; e < 2; ++e) v[e][u] = __ldcg(&from.o[2 * c + e][r]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) next = fmaxf(next, q[u].x);
        const float zero = next == -INFINITY ? 0.f : next, f0 = fast_exp2(top - zero);
        top = next;
        l *= f0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[e].x *= f0; o[e].y *= f0; o[e].z *= f0; o[e].w *= f0;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float w = fast_exp2(q[u].x - zero);      // (0 for a part that is not there; its outputs are another part's)
          l = fmaf(w, q[u].y, l);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            o[e].x = fmaf(w, v[e][u].x, o[e].x);
            o[e].y = fmaf(w, v[e][u].y, o[e].y);
            o[e].z = fmaf(w, v[e][u].z, o[e].z);
            o[e].w = fmaf(w, v[e][u].w, o[e].w);
          }
        }
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t row = s0 + i_seq;
      const int head = hk * heads_all + in_head + h;
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.o) + row * a.o_stride + head * DH + c * 8) =
          make_uint4(pack_16<F16>(o[0].x * inv, o[0].y * inv), pack_16<F16>(o[0].z * inv, o[0].w * inv), pack_16<F16>(o[1].x * inv, o[1].y * inv),
                     pack_16<F16>(o[1].z * inv, o[1].w * inv));
      if (c == 0 && a.lse) a.lse[row * a.n_q_heads + head] = l == 0.f ? -INFINITY : kLn2 * (top + log2f(l));
    }
  }
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

int shared_attention_tile_heads(int n_q_heads, int n_kv_heads) { return std::min(n_q_heads / n_kv_heads, SA_ROWS); }
int shared_attention_tile_seqs(int n_q_heads, int n_kv_heads) { return SA_ROWS / shared_attention_tile_heads(n_q_heads, n_kv_heads); }

cudaError_t shared_attention_set_attributes() {
  for (int i = 0; i < 8; ++i) {
    const int dh = i & 1 ? 128 : 64;
    const cudaError_t e = set_kernel_smem(pick(dh, i & 2, i & 4), dh == 128 ? sa_smem<128>() : sa_smem<64>());
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_shared_attention(const hs_shared_attention_t& a, const CUtensorMap& tm_kv, const CUtensorMap& tm_q, int sm_count, int sm_budget,
                                    cudaStream_t stream) {
  SharedParams p{};
  p.tm_kv = tm_kv;
  p.tm_q = tm_q;
  p.a = a;
  p.score = score_scale(a.scale, a.cap);
  p.heads = shared_attention_tile_heads(a.n_q_heads, a.n_kv_heads);
  p.chunks = (a.n_q_heads / a.n_kv_heads + p.heads - 1) / p.heads;
  p.tile_seqs = shared_attention_tile_seqs(a.n_q_heads, a.n_kv_heads);
  p.shares = share_count(sm_count);
  // Without a cap and slopes the kernel masks and compares raw scores and multiplies by the scale in the exponent: right for a positive scale only.  The other
  // instantiation scales first.
  const bool modified = a.cap > 0.f || a.slopes != nullptr || !(a.scale > 0.f);
  return launch_step_kernel(pick(a.head_dim, a.type == HS_TYPE_F16, modified), std::min(sm_budget, p.shares), SA_THREADS,
                            a.head_dim == 128 ? sa_smem<128>() : sa_smem<64>(), stream, true, p);
}

}  // namespace hs
