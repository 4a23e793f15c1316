// Attention of chunks of new tokens over the paged cache on the 5th-generation tensor cores, with capped scores, a distance bias, a
// sliding window and a prefix; planned on the device.
//
// The pipeline is that of the prefill attention of hs_stage_step (attention_prefill.cu): two Q tiles of 128 rows share the K and V
// blocks of 64 keys, S = Q K^T into tensor memory, one softmax thread per row, P back into tensor memory over S, O += P V.  Its own:
//   work     an item is (sequence, KV head or sixteen of its query heads, two tiles of tokens).  Every block counts the sequences'
//            items in shared memory; the lead producer takes item numbers from a queue and finds their sequence by bisection.
//   keys     an item looks at the blocks of the prefix, then at those from its first row's window to its last row's position.  Rows
//            mask by selection; V rows of keys that no row of the item sees are zeroed, and pages without such a key are not fetched.
//   parts    where a call has few items with many keys, their key blocks are divided among blocks; a part's rows go to the workspace, and the block
//            that delivers a tile's last rows joins its parts, in order, before it leaves.
//   scores   x = cap tanh(scale s / cap) - slope |p - j| in log2 units; tanh is a polynomial while the warp's scores allow it, as
//            the exponentials already take most of their unit's time.
//
// What bounds it is the softmax warps' chain, S read, maximum, exponentials, P written: 64 keys take 2900 cycles of a pair of tiles with a cap, 2100 without, the
// matrix products 45 % of that.  2048 rows at position 4095 behind a prefix, 28 heads on 4 of 128, capped: 166 us, 543 TFLOP/s; without the cap 118.
// Two threads per row (193 us at 169), half of the exponentials as polynomials (200) and tiles half a block apart (no change) were not kept.
#include <math.h>

#include <algorithm>

#include "paged_scores.cuh"

namespace hs {
namespace {

constexpr int PC_THREADS = 448, PC_KEYS = 64, PC_STAGES = 4;
constexpr int PC_TMEM = 512;
constexpr int PC_MIN_BLOCKS = 4, PC_DIVIDED = 12;       // key blocks of a part of an item; of an item that is divided
constexpr float PC_JOIN_FACTOR = 3.f;
constexpr int PC_HEADS = 16;               // query heads of an item at most: eight tokens of each fill a tile
constexpr float kRefSlack = 8.f;           // log2 units by which a row's running maximum may exceed its reference
constexpr float kLn2 = 0.6931471805599453f;

template <int DH>
struct Geom {
  static constexpr int HALVES = DH / 64;
  static constexpr int Q_BYTES = HALVES * 16384;        // one tile: [half][128 rows][128 B]
  static constexpr int KV_BYTES = HALVES * 8192;        // K (or V) of one block: [half][4 pages][16 keys][128 B]
  static constexpr int SMEM = 1024 + 2 * Q_BYTES + 2 * PC_STAGES * KV_BYTES + 1024 + (HS_DEVICE_MAX_SEQS + 1) * 4 + kMaxShares * 4;
  // tensor-memory columns: S(tile, buffer) at tile * 128 + buffer * 64, P over its first 32 columns; O(tile) at 256 + tile * DH
  static constexpr int S0 = 0, O0 = 256;
};
static_assert(Geom<128>::SMEM <= 227 * 1024, "fits one SM");

struct ChunkParams {
  CUtensorMap tm_kv, tm_q;
  hs_paged_attention_t a;
  ScoreScale score;
  int chunks, tile_tokens;                 // groups of heads per KV head; tokens per tile
  int shares;                              // items or parts of items that the device works on at a time
};

// How the items' keys are divided: into parts of `blocks` key blocks, `parts` for the longest.
struct Division {
  int parts, blocks;
};
// A tile's part of an item in the workspace: outputs relative to the row's reference, four coordinates of all rows after one another (threads have a row
// each, and write and read side by side), then (reference in log2 units, sum) per row.
template <int DH>
struct TilePart {
  float4 o[DH / 4][128];
  float2 ml[128];
};

// Geometry of one item, or of one part of it, the same in every role.
struct ItemView {
  int valid;                         // 0: no more items; -1: a part without key blocks
  int seq, head0, hk, heads;         // first query head, KV head, query heads
  int row0, pos0;                    // first token row and its position
  int n_tok_a, n_tok_b;              // tokens of tile A / B (0 = tile absent)
  int kv, prefix, from, end;         // keys of the sequence; seen by some row: j < prefix, or from <= j < end
  int n_prefix, first;               // key blocks 0 .. n_prefix - 1, then first, first + 1, ..
  int item, part, parts_a, parts_b;  // the item's number, which of its parts, and how many each tile has (1: not divided)
  int block0;                        // the part's first key block
  int nblk_a, nblk_b, nblk;          // key blocks per tile and of the part
  template <bool DIVIDED>
  __device__ __forceinline__ int key0(int j) const {
    if (DIVIDED) j += block0;
    return (j < n_prefix ? j : first + j - n_prefix) * PC_KEYS;
  }
  // Whether some row sees key j, a key of the page that begins at k0, every key of the block that begins at k0.
  __device__ __forceinline__ bool sees(int j) const { return j < prefix || (j >= from && j < end); }
  __device__ __forceinline__ bool sees_page(int k0) const { return k0 < prefix || (k0 + 15 >= from && k0 < end); }
  __device__ __forceinline__ bool sees_block(int k0) const {
    return k0 + PC_KEYS <= prefix || ((k0 >= from || from <= prefix) && k0 + PC_KEYS <= max(end, from <= prefix ? prefix : 0));
  }
};
struct Barriers {
  uint64_t q_full, q_empty;
  uint64_t k_full[PC_STAGES], k_empty[PC_STAGES], v_full[PC_STAGES], v_empty[PC_STAGES];
  uint64_t s_full[2][2], p_full[2][2], o_full[2][2];
  uint64_t ring_full[2], ring_empty[2];
  ItemView ring_view[2];
  uint32_t tmem_base;
  int abort_flag, n_joins;
  int warp_sum[PC_THREADS / 32], warp_most[PC_THREADS / 32];
};
static_assert(sizeof(Barriers) <= 1024, "barrier block");

// MN-major 16-bit operand with the 128-byte swizzle: atoms of 64 (MN, contiguous) x 8 (K) elements.
__device__ __forceinline__ uint64_t umma_desc_mnmajor_sw128(uint32_t smem_addr, uint32_t lbo, uint32_t sbo) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr & 0x3ffffu) >> 4);
  d |= static_cast<uint64_t>(lbo >> 4) << 16;
  d |= static_cast<uint64_t>(sbo >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
// D[tmem] (+)= A[tmem] * B[smem]^T
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor of a product of 16-bit operands (both bf16, or both fp16) with fp32 sums.
template <bool F16>
__host__ __device__ constexpr uint32_t idesc_16(int M, int N) {
  const uint32_t bf16 = umma_idesc_bf16_f32(M, N);
  return F16 ? bf16 & ~((1u << 7) | (1u << 10)) : bf16;
}

// The n lowest bits (all for n >= 32, none for n <= 0).
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

template <bool DIVIDED>
__device__ __forceinline__ ItemView make_view(const ChunkParams& p, const int* item_begin, Division div, int idx) {
  ItemView v{};
  const hs_paged_attention_t& a = p.a;
  const int n = a.n_seqs, units = a.n_kv_heads * p.chunks, heads_all = a.n_q_heads / a.n_kv_heads, Mt = p.tile_tokens;
  v.item = idx;
  if (DIVIDED) {
    v.item = idx / div.parts;
    v.part = idx - v.item * div.parts;
  }
  const int pair = v.item / units, unit = v.item - pair * units;
  if (pair >= item_begin[n]) return v;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (item_begin[mid] <= pair) lo = mid;
    else hi = mid;
  }
  const SeqView sv = view_seq(a, lo);
  // a sequence's last tokens, which look at the most keys, come first
  const int tok = (item_begin[lo + 1] - 1 - pair) * 2 * Mt;
  v.valid = 1;
  v.seq = lo;
  v.hk = unit / p.chunks;
  const int in_head = (unit - v.hk * p.chunks) * PC_HEADS;
  v.head0 = v.hk * heads_all + in_head;
  v.heads = min(heads_all - in_head, PC_HEADS);
  v.row0 = sv.row + tok;
  v.pos0 = sv.kv - sv.rows + tok;
  const int n_tok = min(sv.rows - tok, 2 * Mt);
  v.n_tok_a = min(n_tok, Mt);
  v.n_tok_b = n_tok - v.n_tok_a;
  v.kv = sv.kv;
  v.prefix = sv.prefix;
  v.from = a.window > 0 && v.pos0 >= a.window ? v.pos0 - a.window + 1 : 0;
  v.end = max(v.pos0 + n_tok, 0);          // (at most kv, as are prefix and from)
  v.n_prefix = (v.prefix + PC_KEYS - 1) / PC_KEYS;
  v.first = max(v.from / PC_KEYS, v.n_prefix);
  // (at least one block, so that rows that see no key take the same way)
  v.nblk_a = max(v.n_prefix + max((max(v.pos0 + v.n_tok_a, 0) + PC_KEYS - 1) / PC_KEYS - v.first, 0), 1);
  v.nblk_b = v.n_tok_b > 0 ? max(v.n_prefix + max((v.end + PC_KEYS - 1) / PC_KEYS - v.first, 0), 1) : 0;
  v.parts_a = v.parts_b = 1;
  if (DIVIDED && div.parts > 1) {
    v.block0 = v.part * div.blocks;
    v.parts_a = (v.nblk_a + div.blocks - 1) / div.blocks;
    v.parts_b = (v.nblk_b + div.blocks - 1) / div.blocks;
    v.nblk_a = min(max(v.nblk_a - v.block0, 0), div.blocks);
    v.nblk_b = min(max(v.nblk_b - v.block0, 0), div.blocks);
  }
  v.nblk = max(v.nblk_a, v.nblk_b);
  if (DIVIDED && v.nblk == 0) v.valid = -1;
  return v;
}

// Joins the parts of a tile's rows, in order: a thread has a row and some of its coordinates, the fewer the fewer rows there are; eight of them in eight parts
// are on their way at a time.
template <int DH, bool F16>
__device__ __forceinline__ void join_tile(const ChunkParams& p, const ItemView& v, Division div, int t) {
  const hs_paged_attention_t& a = p.a;
  const int n_tok = t ? v.n_tok_b : v.n_tok_a, n_parts = t ? v.parts_b : v.parts_a, n_rows = v.heads * n_tok;
  const int side = (n_rows + 31) & ~31, groups = PC_THREADS / side, group = int(threadIdx.x) / side, q = int(threadIdx.x) - group * side;
  if (q >= n_rows || group >= groups) return;
  const int hg = q / n_tok, tok = q - hg * n_tok, r = hg * p.tile_tokens + tok;
  const TilePart<DH>* tile_parts = reinterpret_cast<const TilePart<DH>*>(static_cast<const char*>(a.workspace) + kWsScratch) + v.item * div.parts * 2 + t;
  float top = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < n_parts; k0 += 8) {
    float2 ml[8];
    float next = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) ml[u] = k0 + u < n_parts ? __ldcg(&tile_parts[2 * (k0 + u)].ml[r]) : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int u = 0; u < 8; ++u) next = fmaxf(next, ml[u].x);
    const float zero = next == -INFINITY ? 0.f : next;
    l *= fast_exp2(top - zero);
#pragma unroll
    for (int u = 0; u < 8; ++u) l = fmaf(fast_exp2(ml[u].x - zero), ml[u].y, l);
    top = next;
  }
  const int64_t row = v.row0 + t * p.tile_tokens + tok;
  const float zero = top == -INFINITY ? 0.f : top, inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = static_cast<uint16_t*>(a.o) + row * a.o_stride + (v.head0 + hg) * DH;
#pragma unroll 1
  for (int c = 2 * group; c < DH / 4; c += 2 * groups) {
    float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
    for (int k0 = 0; k0 < n_parts; k0 += 8) {
      float m[8];
      float4 x[2][8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const bool there = k0 + u < n_parts;
        const TilePart<DH>& from = tile_parts[2 * (k0 + u)];
        m[u] = there ? __ldcg(&from.ml[r].x) : -INFINITY;
#pragma unroll
        for (int e = 0; e < 2; ++e) x[e][u] = there ? __ldcg(&from.o[c + e][r]) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float f = fast_exp2(m[u] - zero);          // (0 for a part that is not there)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[e].x = fmaf(f, x[e][u].x, o[e].x);
          o[e].y = fmaf(f, x[e][u].y, o[e].y);
          o[e].z = fmaf(f, x[e][u].z, o[e].z);
          o[e].w = fmaf(f, x[e][u].w, o[e].w);
        }
      }
    }
    *reinterpret_cast<uint4*>(dst + c * 4) = make_uint4(pack_16<F16>(o[0].x * inv, o[0].y * inv), pack_16<F16>(o[0].z * inv, o[0].w * inv),
                                                       pack_16<F16>(o[1].x * inv, o[1].y * inv), pack_16<F16>(o[1].z * inv, o[1].w * inv));
  }
  if (group == 0 && a.lse) a.lse[row * a.n_q_heads + v.head0 + hg] = l == 0.f ? -INFINITY : kLn2 * (top + log2f(l));
}

template <int DH, bool F16, bool MOD, bool DIVIDED>
__global__ void __launch_bounds__(PC_THREADS, 1) paged_chunk_kernel(const __grid_constant__ ChunkParams p) {
  using G_ = Geom<DH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_smem = smem;                                   // tile A then tile B
  uint8_t* k_smem = q_smem + 2 * G_::Q_BYTES;
  uint8_t* v_smem = k_smem + PC_STAGES * G_::KV_BYTES;
  Barriers* bar = reinterpret_cast<Barriers*>(v_smem + PC_STAGES * G_::KV_BYTES);
  int* item_begin = reinterpret_cast<int*>(reinterpret_cast<uint8_t*>(bar) + 1024);
  int* joins = item_begin + HS_DEVICE_MAX_SEQS + 1;         // [tiles of divided items]: those that this block joins
  volatile int* abort_flag = &bar->abort_flag;
  const hs_paged_attention_t& a = p.a;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int Mt = p.tile_tokens;
  int* queue = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsChunkQueue);

  if (threadIdx.x == 0) {
    mbar_init(&bar->q_full, 1);
    mbar_init(&bar->q_empty, 2);              // one arrival per MMA thread
    for (int i = 0; i < PC_STAGES; ++i) {
      mbar_init(&bar->k_full[i], 2);
      mbar_init(&bar->k_empty[i], 2);
      mbar_init(&bar->v_full[i], 2);
      mbar_init(&bar->v_empty[i], 2);
    }
    for (int t = 0; t < 2; ++t)
      for (int i = 0; i < 2; ++i) {
        mbar_init(&bar->s_full[t][i], 1);
        mbar_init(&bar->p_full[t][i], 128);
        mbar_init(&bar->o_full[t][i], 1);
      }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar->ring_full[i], 1);
      mbar_init(&bar->ring_empty[i], 13);     // eight softmax warps, two MMA warps, three further producers
    }
    bar->abort_flag = 0;
    bar->n_joins = 0;
    fence_barrier_init();
    tma_prefetch_desc(&p.tm_kv);
    tma_prefetch_desc(&p.tm_q);
  }
  if (warp == 9) {
    tmem_alloc(&bar->tmem_base, PC_TMEM);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = bar->tmem_base;
  griddep_wait();
  Division div = {1, 0};
  {
    // the plan: pairs of tiles of all sequences, summed, and the most key blocks that one can have
    const int n = a.n_seqs, per = (n + PC_THREADS - 1) / PC_THREADS, s0 = int(threadIdx.x) * per;
    int mine = 0, most = 1;
    for (int i = 0; i < per && s0 + i < n; ++i) {
      const SeqView v = view_seq(a, s0 + i);
      if (v.error && blockIdx.x == 0) atomicExch(a.status, v.error);
      item_begin[s0 + i] = mine;
      mine += (v.rows + 2 * Mt - 1) / (2 * Mt);
      const int all = (v.kv + PC_KEYS - 1) / PC_KEYS;
      if (DIVIDED && v.rows > 0) most = max(most, a.window > 0 ? min(all, (v.prefix + PC_KEYS - 1) / PC_KEYS + (min(a.window, v.kv) + min(v.rows, 2 * Mt)) / PC_KEYS + 2) : all);
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    if (DIVIDED) most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) {
      bar->warp_sum[warp] = inc;
      if (DIVIDED) bar->warp_most[warp] = most;
    }
    __syncthreads();
    int before = inc - mine, total = 0;
    for (int w = 0; w < PC_THREADS / 32; ++w) {
      if (w < warp) before += bar->warp_sum[w];
      total += bar->warp_sum[w];
      if (DIVIDED) most = max(most, bar->warp_most[w]);
    }
    for (int i = 0; i < per && s0 + i < n; ++i) item_begin[s0 + i] += before;
    if (threadIdx.x == 0) item_begin[n] = total;
    // Where the items are at most half of what the device works on, long ones are divided.  (A part more costs the join about as much as a block: most is
    // gained at the square root.)
    const int items = total * a.n_kv_heads * p.chunks;
    if (DIVIDED && items > 0 && 2 * items <= p.shares && most >= PC_DIVIDED) {
      const int parts = min(p.shares / items, int(sqrtf(PC_JOIN_FACTOR * float(most))));
      div.blocks = max((most + parts - 1) / parts, PC_MIN_BLOCKS);
      div.parts = (most + div.blocks - 1) / div.blocks;
    }
    __syncthreads();
  }

  int rs = 0;
  uint32_t rph = 0;       // item ring slot / phase
  uint32_t n_items_seen = 0;
  uint32_t blk_base = 0;  // key blocks of all earlier items of this thread block (K / V ring position)

  if (warp == 8 || warp >= 11) {
    // ========================================================== TMA producers ==
    // Producer 0 (warp 8) owns the work queue and loads pages 0, 1 of every K block; producer 1 pages 2, 3 of K; producers 2 and 3 the
    // same of V.  All four load the Q tiles.  Lane l holds the id of page l of the current eight key blocks.
    const int pi = warp == 8 ? 0 : warp - 10;           // producer index 0..3
    const int kv = pi >> 1, w0 = (pi & 1) * 2;          // K or V; first of its two pages in a block
    int q_next = int(blockIdx.x);                       // lane 0 of the lead: the next item's number
    ItemView v_next{};
    auto next_view = [&]() {
      v_next = make_view<DIVIDED>(p, item_begin, div, q_next);
      while (DIVIDED && v_next.valid < 0) {                          // (the queue ends)
        q_next = int(gridDim.x) + atomicAdd(queue, 1);
        v_next = make_view<DIVIDED>(p, item_begin, div, q_next);
      }
    };
    if (pi == 0 && lane == 0) next_view();
    for (;;) {
      bool ok = true;
      ItemView v;
      if (pi == 0) {
        if (lane == 0) {
          ok = mbar_wait(&bar->ring_empty[rs], rph ^ 1, abort_flag, a.status);
          if (ok) {
            bar->ring_view[rs] = v_next;
            mbar_arrive(&bar->ring_full[rs]);
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        __syncwarp();
        v = bar->ring_view[rs];
      } else {
        ok = mbar_wait(&bar->ring_full[rs], rph, abort_flag, a.status);
        if (!__all_sync(0xffffffffu, ok)) break;
        v = bar->ring_view[rs];
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->ring_empty[rs]);
      }
      if (++rs == 2) { rs = 0; rph ^= 1; }
      if (!v.valid) break;
      const int32_t* table = a.block_tables + int64_t(v.seq) * a.max_pages_per_seq;
      // page id of page l & 3 of block j0 + l / 4: -1 for a page that no row sees, or outside the pool
      auto page_id = [&](int j0) {
        const int j = j0 + (lane >> 2);
        if (j >= v.nblk) return -1;
        const int k0 = v.template key0<DIVIDED>(j) + (lane & 3) * 16;
        if (!v.sees_page(k0)) return -1;
        const int id = table[k0 >> 4];
        if (id >= 0 && id < a.num_pages) return id;
        atomicExch(a.status, kErrBadBlockTable);
        return -1;
      };
      int pg_next = page_id(0), pg_cur = -1;
      {
        if (lane == 0) ok = mbar_wait(&bar->q_empty, (n_items_seen & 1) ^ 1, abort_flag, a.status);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (ok) {
          const int n_tiles = v.n_tok_b > 0 ? 2 : 1;
          const int n_copies = n_tiles * v.heads * G_::HALVES;
          if (pi == 0 && lane == 0) mbar_expect_tx(&bar->q_full, n_copies * Mt * 128);
          for (int cidx = pi + 4 * lane; cidx < n_copies; cidx += 128) {      // (tile, head, half), half fastest
            const int h = cidx % G_::HALVES, g = (cidx / G_::HALVES) % v.heads, t = cidx / (G_::HALVES * v.heads);
            tma_load_2d(q_smem + t * G_::Q_BYTES + h * 16384 + g * Mt * 128, &p.tm_q, &bar->q_full, (v.head0 + g) * DH + h * 64, v.row0 + t * Mt);
          }
        }
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      ++n_items_seen;
      for (int kb = 0; kb < v.nblk && ok; ++kb) {
        if (pi == 0 && lane == 0) {
          if (kb == max(0, v.nblk - 4)) q_next = int(gridDim.x) + atomicAdd(queue, 1);
          if (kb == v.nblk - 2 && v.nblk > 2) next_view();
        }
        if ((kb & 7) == 0) {
          pg_cur = pg_next;
          pg_next = page_id(kb + 8);
        }
        const uint32_t gb = blk_base + kb;
        const uint32_t st = gb % PC_STAGES, ph = (gb / PC_STAGES) & 1;
        uint64_t* full = kv ? &bar->v_full[st] : &bar->k_full[st];
        uint8_t* dst = (kv ? v_smem : k_smem) + st * G_::KV_BYTES;
        const int id0 = __shfl_sync(0xffffffffu, pg_cur, (kb & 7) * 4 + w0), id1 = __shfl_sync(0xffffffffu, pg_cur, (kb & 7) * 4 + w0 + 1);
        if (lane == 0) {
          ok = mbar_wait(kv ? &bar->v_empty[st] : &bar->k_empty[st], ph ^ 1, abort_flag, a.status);
          if (ok) {
            const int mine = (id0 >= 0) + (id1 >= 0);
            if (mine > 0) mbar_expect_tx(full, mine * G_::HALVES * 2048);
            else mbar_arrive(full);                                  // nothing to fetch, but the block counts on two arrivals
            for (int w = 0; w < 2; ++w) {
              const int id = w ? id1 : id0;
              if (id < 0) continue;
              const int row = (((a.layer * 2 + kv) * a.num_pages + id) * a.n_kv_heads + v.hk) * 16;
              for (int h = 0; h < G_::HALVES; ++h) tma_load_2d(dst + h * 8192 + (w0 + w) * 2048, &p.tm_kv, full, h * 64, row);
            }
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
      }
      if (!ok) break;
      if (pi == 0 && lane == 0 && v.nblk <= 2) next_view();   // (a short item: not before its own requests are out)
      blk_base += v.nblk;
    }
  } else if (warp == 9 || warp == 10) {
    // ============================================================ MMA issuers ==
    // One issuing thread per tile (warp 9: tile A, warp 10: tile B).  The K and V slots and the Q tiles are released by both threads; one with
    // no block to compute arrives without a commit, but only after it has seen the slot filled.
    if (lane == 0) {
      const int t = warp - 9;
      constexpr uint32_t idesc_s = idesc_16<F16>(128, PC_KEYS);
      constexpr uint32_t idesc_pv = idesc_16<F16>(128, DH) | (1u << 16);   // B (= V) is MN-major
      const uint64_t q_desc = umma_desc_kmajor_sw128(smem_u32(q_smem) + t * G_::Q_BYTES);
      const uint64_t k_desc0 = umma_desc_kmajor_sw128(smem_u32(k_smem));
      const uint64_t v_desc0 = umma_desc_mnmajor_sw128(smem_u32(v_smem), 8192, 1024);
      const uint32_t d_o = tmem + G_::O0 + t * DH, s_base = tmem + G_::S0 + t * 128;
      uint32_t g_s = 0, g_pv = 0;        // blocks of this tile whose S / whose P V has been issued, over all items
      bool ok = true;
      auto pv_block = [&](const ItemView& v, int j) -> bool {
        const uint32_t gb = blk_base + j, vst = gb % PC_STAGES;
        if (!mbar_wait(&bar->v_full[vst], (gb / PC_STAGES) & 1, abort_flag, a.status)) return false;
        if (j >= (t ? v.nblk_b : v.nblk_a)) {                                     // nothing of this tile in the block
          mbar_arrive(&bar->v_empty[vst]);
          return true;
        }
        const uint32_t buf = g_pv & 1, bph = (g_pv >> 1) & 1;
        if (!mbar_wait(&bar->p_full[t][buf], bph, abort_flag, a.status)) return false;
        tc_fence_after_sync();
        const uint64_t vdesc = v_desc0 + uint64_t(vst * (G_::KV_BYTES >> 4));
        const uint32_t a_p = s_base + buf * PC_KEYS, acc0 = j == 0 ? 0u : 1u;    // the item's first block overwrites O
#pragma unroll
        for (int pg = 0; pg < 4; ++pg)        // 16 keys (one page) per MMA: 8 columns of P
          umma_ts(d_o, a_p + 8 * pg, vdesc + uint64_t(pg * (2048 >> 4)), idesc_pv, pg != 0 ? 1u : acc0);
        umma_commit(&bar->o_full[t][buf]);
        umma_commit(&bar->v_empty[vst]);
        ++g_pv;
        return true;
      };
      for (;;) {
        if (!mbar_wait(&bar->ring_full[rs], rph, abort_flag, a.status)) break;
        const ItemView v = bar->ring_view[rs];
        mbar_arrive(&bar->ring_empty[rs]);
        if (++rs == 2) { rs = 0; rph ^= 1; }
        if (!v.valid) break;
        const int nblk = (t ? v.nblk_b : v.nblk_a);
        if (!mbar_wait(&bar->q_full, n_items_seen & 1, abort_flag, a.status)) break;
        ++n_items_seen;
        if (nblk == 0) mbar_arrive(&bar->q_empty);
        for (int j = 0; j < v.nblk && ok; ++j) {
          const uint32_t gb = blk_base + j, kst = gb % PC_STAGES;
          if (!mbar_wait(&bar->k_full[kst], (gb / PC_STAGES) & 1, abort_flag, a.status)) { ok = false; break; }
          if (j < nblk) {
            tc_fence_after_sync();
            const uint32_t buf = g_s & 1;
            const uint64_t kdesc = k_desc0 + uint64_t(kst * (G_::KV_BYTES >> 4));
#pragma unroll
            for (int ks = 0; ks < DH / 16; ++ks)
              umma_bf16(s_base + buf * PC_KEYS, q_desc + uint64_t((ks >> 2) * (16384 >> 4) + 2 * (ks & 3)),
                        kdesc + uint64_t((ks >> 2) * (8192 >> 4) + 2 * (ks & 3)), idesc_s, ks != 0);
            umma_commit(&bar->s_full[t][buf]);
            umma_commit(&bar->k_empty[kst]);                        // the K slot, once these scores are computed
            if (j == nblk - 1) umma_commit(&bar->q_empty);          // and the Q tile after the tile's last scores
            ++g_s;
          } else {
            mbar_arrive(&bar->k_empty[kst]);
          }
          if (j > 0) ok = pv_block(v, j - 1);                       // overlaps the softmax of block j
        }
        if (!ok || !pv_block(v, v.nblk - 1)) break;
        blk_base += v.nblk;
      }
    }
  } else {
    // ================================================================ softmax ==
    const int t = warp >> 2;                      // tile of this warp group
    const int r = threadIdx.x & 127;              // row of the tile = TMEM lane
    const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
    const uint32_t s_col = G_::S0 + t * 128, o_col = G_::O0 + t * DH;
    const ScoreScale& sc = p.score;
    uint32_t g = 0;                               // blocks this tile has processed, over all items
    for (;;) {
      bool ok = mbar_wait(&bar->ring_full[rs], rph, abort_flag, a.status);
      if (!__all_sync(0xffffffffu, ok)) break;
      const ItemView v = bar->ring_view[rs];
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->ring_empty[rs]);
      if (++rs == 2) { rs = 0; rph ^= 1; }
      if (!v.valid) break;
      const int nblk = (t ? v.nblk_b : v.nblk_a), n_tok = (t ? v.n_tok_b : v.n_tok_a);
      if (nblk == 0) { blk_base += v.nblk; continue; }            // the item has no tile for this warp group
      const int hg = r / Mt, tok = r - hg * Mt;
      const bool row_valid = hg < v.heads && tok < n_tok;
      // the row sees keys below `prefix`, and lo .. hi (padding rows behave like the tile's last token)
      const int pos = v.pos0 + t * Mt + min(tok, n_tok - 1);
      const int hi = min(max(pos, v.prefix - 1), v.kv - 1), lo = a.window > 0 ? pos - a.window + 1 : 0;
      const float slope = MOD && a.slopes && row_valid ? a.slopes[v.head0 + hg] * 1.4426950408889634f : 0.f;

      float m_ref = -INFINITY, l_run = 0.f;       // (MOD: in log2 units; else of the raw scores, whose scale is positive)
      uint32_t sreg[32], sreg2[32];
      for (int j = 0; j < nblk; ++j, ++g) {
        const uint32_t buf = g & 1, bph = (g >> 1) & 1;
        ok = mbar_wait(&bar->s_full[t][buf], bph, abort_flag, a.status);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after_sync();
        const int key0 = v.template key0<DIVIDED>(j);
        tmem_ld32(tmem + lane_base + s_col + buf * PC_KEYS, sreg);
        tmem_ld32(tmem + lane_base + s_col + buf * PC_KEYS + 32, sreg2);
        tmem_ld_wait();
        // whether this row does not see every key of the block
        const bool masked = key0 + PC_KEYS - 1 > hi || (key0 < lo && key0 + PC_KEYS > v.prefix);
        uint32_t seen1 = 0xffffffffu, seen2 = 0xffffffffu;       // bit e: key key0 + e, key0 + 32 + e
        if (masked) {
          seen1 = first_bits(hi + 1 - key0) & (~first_bits(lo - key0) | first_bits(v.prefix - key0));
          seen2 = first_bits(hi - 31 - key0) & (~first_bits(lo - 32 - key0) | first_bits(v.prefix - 32 - key0));
        }
        auto mask = [&](uint32_t to) {
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            if (!(seen1 & (1u << e))) sreg[e] = to;
            if (!(seen2 & (1u << e))) sreg2[e] = to;
          }
        };
        auto largest = [&]() {                        // four chains
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
        // Of a capped block that the whole warp sees, the polynomial of the largest score is the largest polynomial, and the reference is part of its
        // last multiply-add: nothing is written back in between.  A mask or a bias has to be applied in between.
        float mx;
        int direct = 0;                               // 3, 5: such a block, by the polynomial's degree; 0: the registers hold finished scores
        if (MOD) {
          int degree = 0;
          bool all_seen = false;
          float top = 0.f;
          if (sc.out != 0.f) {
            if (masked) mask(0u);                     // (what is not seen must not decide which polynomial the others take)
            top = largest();
            const float low = smallest(), u = row_valid ? fmaxf(top * top, low * low) : 0.f;         // (rows of padding hold anything)
            // one vote: the worst row's polynomial (6: degree three, 4: five, 0: none), 1 more where nothing is masked
            const unsigned vote = __reduce_and_sync(0xffffffffu, (u <= sc.limit3 ? 6u : u <= sc.limit5 ? 4u : 0u) | (masked ? 0u : 1u));
            degree = vote >= 6 ? 3 : vote >= 4 ? 5 : 0;
            all_seen = vote & 1u;
          }
          if (degree != 0 && a.slopes == nullptr && all_seen) {
            direct = degree;
            float unused;
            if (degree == 3) split(odd_poly(f2(top, top), sc.c3, f2(0.f, 0.f)), mx, unused);
            else split(odd_poly(f2(top, top), sc.c5, f2(0.f, 0.f)), mx, unused);
          } else {
            // (the distance of a key in front of the row needs its sign only where there is one)
            const float dist = float(pos - key0);
            const bool ahead = pos - key0 < PC_KEYS - 1;
            const F2 base2 = f2(-slope * dist, -slope * dist), slope2 = f2(slope, slope), in2 = f2(sc.in, sc.in);
            auto finish = [&](auto score) {           // score(pair of raw scores, what to add)
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
            if (ahead && slope != 0.f) {              // keys behind the row's position (a prefix): their distance counts the other way
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float f1 = fmaxf(float(e) - dist, 0.f), f3 = fmaxf(float(e + 32) - dist, 0.f);
                sreg[e] = __float_as_uint(fmaf(-2.f * slope, f1, __uint_as_float(sreg[e])));
                sreg2[e] = __float_as_uint(fmaf(-2.f * slope, f3, __uint_as_float(sreg2[e])));
              }
            }
            if (masked) mask(0xff800000u);          // -infinity
            mx = largest();
          }
        } else {
          if (masked) mask(0xff800000u);          // -infinity
          mx = largest();
        }
        // the reference maximum moves only when the block's maximum is far above it
        const float unit = MOD ? 1.f : sc.in;
        float alpha = 1.f;
        const bool move = row_valid && mx > -INFINITY && (m_ref == -INFINITY || (mx - m_ref) * unit > kRefSlack);
        if (move) {
          alpha = m_ref == -INFINITY ? 0.f : fast_exp2((m_ref - mx) * unit);
          m_ref = mx;
        }
        const bool rescale = j > 0 && __any_sync(0xffffffffu, move);
        const float neg_ms = m_ref == -INFINITY ? 0.f : -m_ref * unit;
        const F2 neg2 = f2(neg_ms, neg_ms), unit2 = f2(unit, unit);
        F2 sums[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
        uint32_t pk[32];
        auto weights = [&](auto score) {              // score(pair of raw or finished scores) = log2 of their weights
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
            // (at most 2^kRefSlack, rounded once for the product with v; the sums keep fp32.  Against 64 bits that makes 0.0022 of the outputs' spread
            // in bf16 of the 0.0017 that rounding o alone leaves, 0.0002 of 0.0002 in fp16)
            pk[e >> 1] = pack_16<F16>(x0, x1);
            pk[16 + (e >> 1)] = pack_16<F16>(y0, y1);
          }
        };
        if (!MOD) weights([&](F2 s) { return fma2(s, unit2, neg2); });
        else if (direct == 3) weights([&](F2 s) { return odd_poly(s, sc.c3, neg2); });
        else if (direct == 5) weights([&](F2 s) { return odd_poly(s, sc.c5, neg2); });
        else weights([&](F2 s) { return add2(s, neg2); });
        float sum_a, sum_b;
        split(add2(sums[0], sums[1]), sum_a, sum_b);
        const float sum = sum_a + sum_b;
        l_run = l_run * alpha + sum;
        if (rescale) {
          // O must be at rest: the P V product of the previous block has completed (its successor cannot be issued
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
        // P over the first 32 columns of the S buffer just read: column c of row r = keys 2 c, 2 c + 1
        tmem_st32(tmem + lane_base + s_col + buf * PC_KEYS, pk);
        // V rows of keys that no row of the item sees may hold anything and must not meet the weight 0
        if (!v.sees_block(key0)) {
          const uint32_t gb = blk_base + j, s = gb % PC_STAGES;
          const bool w = mbar_wait(&bar->v_full[s], (gb / PC_STAGES) & 1, abort_flag, a.status);
          if (!__all_sync(0xffffffffu, w)) { ok = false; break; }
          uint8_t* vst = v_smem + s * G_::KV_BYTES;
          for (int idx = r; idx < PC_KEYS * G_::HALVES * 8; idx += 128) {
            const int u = idx & 7, h = (idx >> 3) % G_::HALVES, k = (idx >> 3) / G_::HALVES;
            if (v.sees(key0 + k)) continue;
            *reinterpret_cast<uint4*>(vst + h * 8192 + (k >> 4) * 2048 + (k & 15) * 128 + (u << 4)) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
        }
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(&bar->p_full[t][buf]);
      }
      if (!ok) break;
      // the item's last P V product, then the tile's rows of O leave through registers
      ok = mbar_wait(&bar->o_full[t][(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag, a.status);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after_sync();
      const int64_t row = v.row0 + t * Mt + tok;
      uint16_t* dst = static_cast<uint16_t*>(a.o) + row * a.o_stride + (v.head0 + hg) * DH;
      // (a rounding of its own, so that both instantiations give a row the same bits: left to itself the compiler fuses it into lse's sum in one of them)
      const float m_log2 = MOD ? m_ref : __fmul_rn(m_ref, sc.in);
      if (!DIVIDED || (t ? v.parts_b : v.parts_a) == 1) {
        const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
        if (row_valid && a.lse) a.lse[row * a.n_q_heads + v.head0 + hg] = l_run == 0.f ? -INFINITY : kLn2 * (m_log2 + log2f(l_run));
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) {
          tmem_ld32(tmem + lane_base + o_col + c * 32, sreg);
          tmem_ld_wait();
          if (row_valid) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = pack_16<F16>(__uint_as_float(sreg[2 * e]) * inv, __uint_as_float(sreg[2 * e + 1]) * inv);
#pragma unroll
            for (int u = 0; u < 4; ++u) *reinterpret_cast<uint4*>(dst + c * 32 + u * 8) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
          }
        }
      } else {
        // A part: its rows go to the workspace.  The block that delivers a tile's last rows joins them before it leaves.
        TilePart<DH>* tile_parts = reinterpret_cast<TilePart<DH>*>(static_cast<char*>(a.workspace) + kWsScratch) + v.item * div.parts * 2 + t;
        TilePart<DH>& mine = tile_parts[2 * v.part];
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) {
          tmem_ld32(tmem + lane_base + o_col + c * 32, sreg);
          tmem_ld_wait();
          if (row_valid) {
#pragma unroll
            for (int u = 0; u < 8; ++u)
              __stcg(&mine.o[c * 8 + u][r], make_float4(__uint_as_float(sreg[4 * u]), __uint_as_float(sreg[4 * u + 1]), __uint_as_float(sreg[4 * u + 2]),
                                                         __uint_as_float(sreg[4 * u + 3])));
          }
        }
        if (row_valid) __stcg(&mine.ml[r], make_float2(m_ref == -INFINITY ? -INFINITY : m_log2, l_run));
        __threadfence();
        __syncwarp();
        if (lane == 0) {
          int* done = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsChunkDone) + v.item * 2 + t;
          if (atomicAdd(done, 1) == 4 * (t ? v.parts_b : v.parts_a) - 1) {           // (one for each warp)
            *done = 0;                                   // ready for the next call
            joins[atomicAdd(&bar->n_joins, 1)] = v.item * 2 + t;
          }
        }
      }
      tc_fence_before_sync();
      blk_base += v.nblk;
    }
  }

  // --------------------------------------------------------------- teardown --
  __syncwarp();
  if (*abort_flag) drain_after_abort();
  tc_fence_before_sync();
  __syncthreads();
  if (DIVIDED && bar->n_joins > 0) {
    __threadfence();
#pragma unroll 1
    for (int i = 0; i < bar->n_joins; ++i) join_tile<DH, F16>(p, make_view<DIVIDED>(p, item_begin, div, (joins[i] >> 1) * div.parts), div, joins[i] & 1);
  }
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, PC_TMEM);
  }
  // the last block to leave puts the queue back to zero
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(queue + 1, 1) == int(gridDim.x) - 1) {
      queue[0] = 0;
      queue[1] = 0;
    }
  }
}

template <int DH>
constexpr int pc_smem() {
  return Geom<DH>::SMEM > kMinSmemBytes ? Geom<DH>::SMEM : kMinSmemBytes;
}
static_assert(kWsChunkQueue + 8 <= kWsChunkDone, "two words");
static_assert(kWsChunkDone + kMaxShares * 4 <= kWsScratch, "a word for both tiles of every divided item");
static_assert(size_t(kMaxShares) * 2 * sizeof(TilePart<128>) <= kWsScratchBytes, "two tiles of every part");

using ChunkKernel = void (*)(ChunkParams);
template <int DH, bool DIVIDED>
ChunkKernel pick(bool f16, bool mod) {
  if (f16) return mod ? paged_chunk_kernel<DH, true, true, DIVIDED> : paged_chunk_kernel<DH, true, false, DIVIDED>;
  return mod ? paged_chunk_kernel<DH, false, true, DIVIDED> : paged_chunk_kernel<DH, false, false, DIVIDED>;
}
ChunkKernel pick(int dh, bool f16, bool mod, bool divided) {
  if (dh == 128) return divided ? pick<128, true>(f16, mod) : pick<128, false>(f16, mod);
  return divided ? pick<64, true>(f16, mod) : pick<64, false>(f16, mod);
}

}  // namespace

int paged_chunk_tile_tokens(int n_q_heads, int n_kv_heads) {
  const int heads = std::min(n_q_heads / n_kv_heads, PC_HEADS);
  return (128 / heads) & ~7;
}

cudaError_t paged_chunk_set_attributes() {
  for (int i = 0; i < 16; ++i) {
    const int dh = i & 1 ? 128 : 64;
    const cudaError_t e = set_kernel_smem(pick(dh, i & 2, i & 4, i & 8), dh == 128 ? pc_smem<128>() : pc_smem<64>());
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_paged_chunk(const hs_paged_attention_t& a, const CUtensorMap& tm_kv, const CUtensorMap& tm_q, int sm_count, int sm_budget, cudaStream_t stream) {
  ChunkParams p{};
  p.shares = share_count(sm_count);
  p.tm_kv = tm_kv;
  p.tm_q = tm_q;
  p.a = a;
  p.score = score_scale(a.scale, a.cap);
  const int heads = a.n_q_heads / a.n_kv_heads;
  p.chunks = (heads + PC_HEADS - 1) / PC_HEADS;
  p.tile_tokens = paged_chunk_tile_tokens(a.n_q_heads, a.n_kv_heads);
  // The kernel that can divide items is taken where every call of this shape has few of them.  (What it carries for that costs it 1 to 6 % on
  // items that are not divided: two chunks of 614 tokens, 28 heads on 4, 29.1 / 31.0 us.)
  const int64_t tokens = 2 * p.tile_tokens;
  const int64_t pairs = std::min(int64_t(a.n_seqs) * ((a.max_q_len + tokens - 1) / tokens), a.n_tokens / tokens + a.n_seqs);
  const bool divided = 2 * pairs * a.n_kv_heads * p.chunks <= p.shares && int64_t(a.max_pages_per_seq) * HS_PAGE_SIZE > (PC_DIVIDED - 1) * PC_KEYS;
  // Without a cap and slopes the kernel masks and compares raw scores and multiplies by the scale in the exponent: right for a positive scale only.  The other
  // instantiation scales first.
  const bool modified = a.cap > 0.f || a.slopes != nullptr || !(a.scale > 0.f);
  return launch_step_kernel(pick(a.head_dim, a.type == HS_TYPE_F16, modified, divided), sm_budget, PC_THREADS,
                            a.head_dim == 128 ? pc_smem<128>() : pc_smem<64>(), stream, true, p);
}

}  // namespace hs
