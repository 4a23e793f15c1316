// Pages that several rows of block tables hold: rows that continue other rows, copies of pages, a pool that is made smaller.
//
// Fork.  Row i becomes what row parent[i] was.  With children_p the rows that name p, a full page of row p loses one holder and gains children_p:
//     shares[page] += children_p - 1,   and a page whose count falls below zero has no holder left
// (a count is the holders but the first; partial sums never fall below it while a holder goes on, so the addition that takes it below zero is the
// only one of its page).  Everything else follows from parent and ctx_len alone, so every block works it out for itself: children, first successors, the copies'
// places on the stack by one running sum.  The tables are changed in place: a block has eight columns of all rows in shared memory before it writes
// them, so no block waits for another; the last one to end sweeps the bits of freed pages, in order, onto the stack.  Rows that share a page in a column
// are neighbours as a rule (beams of a request): a warp adds up their counts first, mostly to zero, which spares the atomics on a prompt's pages.
// Latency bounds it: launch, one round trip for lengths, parents and table entries together, one for the counts, one for the blocks that are done, one for the
// freed pages' bits.  16 rows of 49 pages 7.1 us, 512 rows of 258 pages 11.5 us.
//
// Copy.  A warp takes one head of one page and layer, K or V, at a time: up to 16 rows that follow one another, eight 16-byte pieces a lane on their way.  The pages of a
// layer follow one another, so that what is being copied lies together.  HBM bounds it: 300 whole pages of 28 layers (550 MB read and written) 104 us, 5.3 TB/s; with
// streaming loads and stores it was 108.
//
// Compact.  Bits of the free pages; running sums of the bits number the free pages below the bound and the used ones above it; then tables, counts, stack and
// copy list from those numbers.  Three small kernels, one after the other: each needs the whole of the one in front.  200,000 pages 13.3 us, which is their launches and a few
// round trips each.  A small pool is one block's work, in shared memory: 1,000 pages 5 us.
#include <algorithm>

#include "block_scan.cuh"
#include "device_ops.h"
#include "ptx.cuh"

namespace hs {
namespace {

constexpr int SP_THREADS = 1024, SP_PER_THREAD = HS_DEVICE_MAX_SEQS / SP_THREADS;
constexpr int SP_COLUMNS = 8;                            // columns of a block's slice
constexpr int SP_SMALL_PAGES = 8192, SP_SMALL_WORK = 12288;              // pages that one block compacts at most, and with the entries of tables
constexpr int SP_SMALL_SMEM = 3 * SP_SMALL_PAGES * 4;
constexpr int SP_FORK_SMEM = HS_DEVICE_MAX_SEQS * (6 * 4 + SP_COLUMNS * 4);
static_assert(SP_FORK_SMEM <= 227 * 1024, "fits one SM");
static_assert(HS_BEAMS_MAX_PAGES % 32 == 0 && HS_COMPACT_MAX_PAGES <= HS_BEAMS_MAX_PAGES, "a bit per page");

__device__ __forceinline__ unsigned* page_bits(void* workspace) { return reinterpret_cast<unsigned*>(static_cast<char*>(workspace) + kWsPageBits); }
__device__ __forceinline__ int owned_pages(int ctx) { return (ctx + HS_PAGE_SIZE - 1) / HS_PAGE_SIZE; }

// Where a block has column c of its slice of row i: a column of 32 rows and all columns of four rows both touch every bank once.
__device__ __forceinline__ int entry_of(int i, int c) { return i * SP_COLUMNS + (c ^ (i >> 2 & (SP_COLUMNS - 1))); }

__global__ void __launch_bounds__(SP_THREADS, 1) fork_pages_kernel(const hs_fork_pages_t a) {
  extern __shared__ int smem[];
  __shared__ unsigned long long warp_sums[32];
  __shared__ int most, ended;
  griddep_wait();
  const int n = a.n_rows, tid = threadIdx.x, lane = tid & 31, width = a.max_pages_per_seq;
  int* ctx = smem;                                       // [n] each, as they were
  int* parent = smem + n;
  int* children = smem + 2 * n;
  int* first = smem + 3 * n;                             // successor
  int* place = smem + 4 * n;                             // of the row's copy among the copies, -1: none
  int* target = smem + 5 * n;                            // and its page
  int* slice = smem + 6 * n;                             // [n][SP_COLUMNS]
  // Everything that needs no other answer is asked for at once: counts, lengths, parents, and the first columns whether rows own them or not.
  auto load_slice = [&](int c0) {
#pragma unroll 4
    for (int x = tid; x < n * SP_COLUMNS; x += SP_THREADS) {
      const int i = x / SP_COLUMNS, c = c0 + x % SP_COLUMNS;
      slice[entry_of(i, x % SP_COLUMNS)] = c < width ? a.block_tables[int64_t(i) * width + c] : -1;
    }
  };
  const int free_count = *a.free_count;
  int lengths[SP_PER_THREAD], parents[SP_PER_THREAD];
#pragma unroll
  for (int u = 0; u < SP_PER_THREAD; ++u) {
    const int i = tid + u * SP_THREADS;
    lengths[u] = i < n ? a.ctx_len[i] : 0;
    parents[u] = i < n ? a.parent[i] : -1;
  }
  load_slice(int(blockIdx.x) * SP_COLUMNS);
  if (tid == 0) most = 0;
  for (int i = tid; i < n; i += SP_THREADS) {
    children[i] = 0;
    first[i] = n;
  }
  __syncthreads();
  int wrong = 0;
#pragma unroll
  for (int u = 0; u < SP_PER_THREAD; ++u) {
    const int i = tid + u * SP_THREADS, c = lengths[u], p = parents[u];
    if (i >= n) continue;
    if (c < 0 || c > row_tokens(width) || p < -1 || p >= n) wrong = 1;
    ctx[i] = c;
    parent[i] = p;
    if (p >= 0 && p < n) {
      atomicAdd(&children[p], 1);
      atomicMin(&first[p], i);
    }
    if (!wrong) atomicMax(&most, owned_pages(c));
  }
  wrong = __syncthreads_or(wrong);
  unsigned long long mine = 0, n_copies = 0;
  if (!wrong) {
#pragma unroll
    for (int u = 0; u < SP_PER_THREAD; ++u) {
      const int i = tid * SP_PER_THREAD + u;
      if (i >= n) continue;
      const int p = parent[i];
      place[i] = p >= 0 && ctx[p] % HS_PAGE_SIZE != 0 && first[p] != i ? 0 : -1;
      mine += place[i] == 0 ? 1 : 0;
    }
  }
  unsigned long long at = block_scan(mine, warp_sums, n_copies);
  const int error = wrong || free_count < 0 || free_count > a.num_pages ? kErrInvalidArg : int(n_copies) > free_count ? kErrOutOfPages : 0;
  if (error) {
    for (int i = int(blockIdx.x) * SP_THREADS + tid; i < n; i += int(gridDim.x) * SP_THREADS) {
      a.copy_src[i] = a.copy_dst[i] = -1;
      a.copy_len[i] = 0;
    }
    if (blockIdx.x == 0 && tid == 0) atomicExch(a.status, error);
    return;
  }
#pragma unroll
  for (int u = 0; u < SP_PER_THREAD; ++u) {
    const int i = tid * SP_PER_THREAD + u;
    if (i >= n) continue;
    if (place[i] == 0) {
      target[i] = a.free_list[free_count - 1 - int(at)];
      place[i] = int(at++);
    } else if (blockIdx.x == 0) {
      a.copy_src[i] = a.copy_dst[i] = -1;
      a.copy_len[i] = 0;
    }
  }

  unsigned* bits = page_bits(a.workspace);
  int* word = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsTables);         // blocks that are done, and in its upper half those that freed a page
  bool bad_page = false, freed = false;
  auto inside = [&](int page) { return page >= 0 && page < a.num_pages; };
  for (int c0 = int(blockIdx.x) * SP_COLUMNS; c0 < most; c0 += int(gridDim.x) * SP_COLUMNS) {
    if (c0 >= int(gridDim.x) * SP_COLUMNS) load_slice(c0);
    for (int x = tid; x < n * SP_COLUMNS; x += SP_THREADS)               // (a thread's own entries)
      if (c0 + x % SP_COLUMNS >= owned_pages(ctx[x / SP_COLUMNS])) slice[entry_of(x / SP_COLUMNS, x % SP_COLUMNS)] = -1;
    __syncthreads();
    // A warp takes a column of 32 rows; the first of neighbours with the same page adds for all of them: a difference of running sums.
    // (Four of them at a time, so that the counts' answers are waited for once.)
    for (int x0 = tid >> 5; x0 < (n + 31) / 32 * SP_COLUMNS; x0 += 4 * (SP_THREADS / 32)) {
      int pages[4], by[4], was[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int x = x0 + u * (SP_THREADS / 32), i = x / SP_COLUMNS * 32 + lane, c = c0 + x % SP_COLUMNS;
        by[u] = pages[u] = 0;
        if (x / SP_COLUMNS * 32 >= n) continue;          // (the same for the whole warp)
        const bool owned = i < n && c < owned_pages(ctx[i]);
        const int page = i < n ? slice[entry_of(i, x % SP_COLUMNS)] : -1;             // (entries that a row does not own are -1 here)
        bad_page |= owned && !inside(page);
        // holders that full pages gain and lose; a last page that is not full is lost by a row that nobody continues
        int sum = !owned ? 0 : c < ctx[i] / HS_PAGE_SIZE ? children[i] - 1 : children[i] == 0 ? -1 : 0;
        const int mine = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, sum, o);
          sum += lane >= o ? y : 0;
        }
        const int before = __shfl_up_sync(0xffffffffu, page, 1);
        const bool leads = lane == 0 || page != before;
        const unsigned behind = __ballot_sync(0xffffffffu, leads) & (0xfffffffeu << lane);
        const int run = __shfl_sync(0xffffffffu, sum, behind ? __ffs(behind) - 2 : 31) - (sum - mine);
        pages[u] = page;
        by[u] = leads && inside(page) ? run : 0;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) was[u] = by[u] != 0 ? atomicAdd(&a.shares[pages[u]], by[u]) : -1;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (was[u] < 0 || was[u] + by[u] >= 0) continue;
        atomicOr(&bits[pages[u] >> 5], 1u << (pages[u] & 31));
        freed = true;
      }
    }
    for (int x = tid; x < n * SP_COLUMNS; x += SP_THREADS) {
      const int i = x / SP_COLUMNS, c = c0 + x % SP_COLUMNS, p = parent[i];
      int32_t* entry = a.block_tables + int64_t(i) * width + c;
      if (p < 0 || c >= owned_pages(ctx[p])) {
        if (c < owned_pages(ctx[i])) *entry = -1;
        continue;
      }
      int page = slice[entry_of(p, x % SP_COLUMNS)];
      if (place[i] >= 0 && c == ctx[p] / HS_PAGE_SIZE) {
        const int from = page;
        page = target[i];
        const bool ok = inside(from) && inside(page);
        bad_page |= !ok;
        a.copy_src[i] = ok ? from : -1;
        a.copy_dst[i] = ok ? page : -1;
        a.copy_len[i] = ok ? ctx[p] % HS_PAGE_SIZE : 0;
      }
      if (page != slice[entry_of(i, x % SP_COLUMNS)] || page == -1) *entry = page;
    }
    __syncthreads();
  }
  if (bad_page) atomicExch(a.status, kErrBadBlockTable);
  const int any = __syncthreads_or(freed);
  if (tid == 0) {
    __threadfence();
    const int now = atomicAdd(word, any ? 0x10001 : 1) + (any ? 0x10001 : 1);
    ended = (now & 0xffff) == int(gridDim.x) ? now : 0;
    __threadfence();
  }
  __syncthreads();
  if (!ended) return;
  for (int i = tid; i < n; i += SP_THREADS) {
    const int p = parent[i];
    a.ctx_len[i] = p >= 0 ? ctx[p] : 0;
  }
  int top = free_count - int(n_copies);
  if (ended >> 16) {
    // freed pages in rising order, four words a thread
    const int n_words = (a.num_pages + 31) / 32;
    uint4* words = reinterpret_cast<uint4*>(bits);
    for (int w0 = 0; w0 < n_words; w0 += 4 * SP_THREADS) {
      const int at = w0 / 4 + tid;
      const uint4 q = 4 * at < n_words ? __ldcg(words + at) : make_uint4(0, 0, 0, 0);
      const unsigned long long count = __popc(q.x) + __popc(q.y) + __popc(q.z) + __popc(q.w);
      unsigned long long total;
      int to = top + int(block_scan(count, warp_sums, total));
      if (count > 0) {
        words[at] = make_uint4(0, 0, 0, 0);              // ready for the next call
        const unsigned left4[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          for (unsigned left = left4[e]; left; left &= left - 1) {
            const int page = (4 * at + e) * 32 + __ffs(left) - 1;
            a.shares[page] = 0;
            if (to < a.num_pages) a.free_list[to] = page;
            ++to;
          }
        }
      }
      top += int(total);
      __syncthreads();                                   // (warp_sums)
    }
    top = min(top, a.num_pages);
  }
  if (tid == 0) {
    *a.free_count = top;
    *word = 0;                                           // ready for the next call
  }
}

// ------------------------------------------------------------------------------------------------------------ copies
constexpr int CP_THREADS = 1024, CP_UNROLL = 8;

__global__ void __launch_bounds__(CP_THREADS, 1) copy_pages_kernel(const hs_copy_pages_t a) {
  const int lane = threadIdx.x & 31;
  const int pieces = a.head_dim / 8;                     // of a token
  const int units = a.n_layers * 2 * a.n_kv_heads, n = a.n_copies * units;
  const int stride = int(gridDim.x) * (CP_THREADS / 32);
  uint4* pool = static_cast<uint4*>(a.kv_pool);
  griddep_wait();
  // A warp's heads follow one another in steps of the grid: neighbouring warps have neighbouring heads of a page.
  for (unsigned x = blockIdx.x * (CP_THREADS / 32) + (threadIdx.x >> 5); x < unsigned(n); x += unsigned(stride)) {
    const int rest = int(x) / a.n_kv_heads, head = int(x) - rest * a.n_kv_heads, layer = rest / a.n_copies, i = rest - layer * a.n_copies;
    const int src = a.src[i], dst = a.dst[i], tokens = a.length ? a.length[i] : HS_PAGE_SIZE;
    if (src == -1 || dst == -1) continue;
    if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages || tokens < 0 || tokens > HS_PAGE_SIZE) {
      if (lane == 0) atomicExch(a.status, tokens < 0 || tokens > HS_PAGE_SIZE ? kErrInvalidArg : kErrBadBlockTable);
      continue;
    }
    const int64_t block = int64_t(HS_PAGE_SIZE) * pieces;             // pieces of one head of a page
    const uint4* from = pool + ((int64_t(layer) * a.num_pages + src) * a.n_kv_heads + head) * block;
    uint4* to = pool + ((int64_t(layer) * a.num_pages + dst) * a.n_kv_heads + head) * block;
    const int count = tokens * pieces;
    for (int at = 0; at < count; at += 32 * CP_UNROLL) {
      uint4 v[CP_UNROLL];
#pragma unroll
      for (int u = 0; u < CP_UNROLL; ++u)
        if (at + 32 * u + lane < count) v[u] = from[at + 32 * u + lane];
#pragma unroll
      for (int u = 0; u < CP_UNROLL; ++u)
        if (at + 32 * u + lane < count) to[at + 32 * u + lane] = v[u];
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ compaction
// What the kernels of one call leave one another in the workspace.
struct Compaction {
  int moves, low, free_pages, wrong;                     // used pages from n_keep up; free ones below; all free ones; whether something is wrong
};
__device__ __forceinline__ Compaction* plan_of(const hs_compact_pages_t& a) { return reinterpret_cast<Compaction*>(static_cast<char*>(a.workspace) + kWsScratch); }
__device__ __forceinline__ int* targets_of(const hs_compact_pages_t& a) { return reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsScratch + 256); }      // [n_keep]
__device__ __forceinline__ int* numbers_of(const hs_compact_pages_t& a) { return targets_of(a) + a.n_keep; }        // [num_pages - n_keep]: of a move, -1 for a free page
__device__ __forceinline__ int* sources_of(const hs_compact_pages_t& a) { return targets_of(a) + a.num_pages; }     // [num_pages - n_keep]
static_assert(256 + size_t(HS_COMPACT_MAX_PAGES) * 2 * sizeof(int) <= kWsScratchBytes, "three lists of pages");

// The bits of the free pages, from the stack.
__device__ __forceinline__ void mark_free(const hs_compact_pages_t& a, int free_count, unsigned* bits, int first, int stride) {
  const int n = free_count < 0 || free_count > a.num_pages ? 0 : free_count;
#pragma unroll 4
  for (int i = first; i < n; i += stride) {
    const int page = a.free_list[i];
    if (page >= 0 && page < a.num_pages) atomicOr(&bits[page >> 5], 1u << (page & 31));
  }
}

// Numbers the pages of words b0 .. b1 - 1 by the whole block: counts of free pages below the bound (upper half) and used ones from it up, those in front of b0 in `before`.
// Returns the counts behind b1 - 1.  LOAD reads a word of the bits.
template <typename F>
__device__ __forceinline__ unsigned long long number_pages(const hs_compact_pages_t& a, F load, int b0, int b1, unsigned long long before, unsigned long long* warp_sums, int* targets,
                                                           int* numbers, int* sources) {
  const int tid = threadIdx.x, keep = a.n_keep;
  auto below = [&](int w) { return keep <= w * 32 ? 0u : keep >= w * 32 + 32 ? ~0u : (1u << (keep - w * 32)) - 1u; };
  auto exists = [&](int w) { return a.num_pages >= w * 32 + 32 ? ~0u : (1u << (a.num_pages - w * 32)) - 1u; };
  // a warp a run of words, a lane a page of each
  const int lane = tid & 31, per = (b1 - b0 + 31) / 32, w0 = min(b0 + (tid >> 5) * per, b1), w1 = min(w0 + per, b1);
  unsigned long long mine = 0, total = 0;
  for (int w = w0 + lane; w < w1; w += 32) {
    const unsigned free = load(w);
    mine += (static_cast<unsigned long long>(__popc(free & below(w))) << 32) + __popc(~free & ~below(w) & exists(w));
  }
  const unsigned long long at = __shfl_sync(0xffffffffu, before + block_scan(mine, warp_sums, total), 0);
  int low = int(at >> 32), number = int(unsigned(at));
  const unsigned in_front = (1u << lane) - 1u;
#pragma unroll 2
  for (int w = w0; w < w1; ++w) {
    const unsigned free = load(w), free_low = free & below(w), high = ~below(w) & exists(w), used = high & ~free;
    const int page = w * 32 + lane;
    if (free_low >> lane & 1u) targets[low + __popc(free_low & in_front)] = page;
    if (high >> lane & 1u) {
      const int n = number + __popc(used & in_front);
      const bool moves = used >> lane & 1u;
      numbers[page - keep] = moves ? n : -1;
      if (moves) sources[n] = page;
    }
    low += __popc(free_low);
    number += __popc(used);
  }
  return before + total;
}

__device__ __forceinline__ Compaction compaction_of(const hs_compact_pages_t& a, unsigned long long end, int wrong) {
  const int moves = int(unsigned(end)), low = int(end >> 32);
  return Compaction{moves, low, low + (a.num_pages - a.n_keep - moves), wrong};
}

// Copy list, counts, stack and tables, by threads first, first + stride, ...
__device__ __forceinline__ void move_pages(const hs_compact_pages_t& a, const Compaction& plan, int free_count, const int* targets, const int* numbers, const int* sources, int first,
                                           int stride) {
  const int keep = a.n_keep;
  const int error = plan.wrong || plan.free_pages != free_count || plan.moves > a.max_copies ? kErrInvalidArg : plan.moves > plan.low ? kErrOutOfPages : 0;
  const int moves = error ? 0 : plan.moves;
  for (int k = first; k < a.max_copies; k += stride) {
    a.copy_src[k] = k < moves ? sources[k] : -1;
    a.copy_dst[k] = k < moves ? targets[k] : -1;
  }
  if (error) {
    if (first == 0) atomicExch(a.status, error);
    return;
  }
  for (int k = first; k < moves; k += stride) {
    a.shares[targets[k]] = a.shares[sources[k]];
    a.shares[sources[k]] = 0;
  }
  // the highest free page at the bottom of the stack
  const int low = plan.low - moves, high = a.num_pages - keep;
  for (int k = first; k < low + high; k += stride) a.free_list[low + high - 1 - k] = k < low ? targets[moves + k] : keep + k - low;
  // a warp a row's run of entries, four of them at a time, whose loads do not wait for one another
  const int lane = threadIdx.x & 31, width = (a.max_pages_per_seq + 31) / 32;
  const int64_t runs = int64_t(a.n_rows) * width;
  bool bad_page = false;
  for (int64_t x0 = first >> 5; x0 < runs; x0 += 4 * (stride >> 5)) {
    int32_t* entry[4];
    int page[4], owned[4], c[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t x = x0 + u * (stride >> 5);
      const int row = int(min(x, runs - 1) / width);
      c[u] = int(x - int64_t(row) * width) * 32 + lane;
      entry[u] = a.block_tables + int64_t(row) * a.max_pages_per_seq + c[u];
      const bool there = x < runs && c[u] < a.max_pages_per_seq;
      page[u] = there ? *entry[u] : 0;
      owned[u] = there ? owned_pages(a.ctx_len[row]) : 0;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c[u] >= owned[u]) continue;
      if (page[u] < 0 || page[u] >= a.num_pages) {
        bad_page = true;
      } else if (page[u] >= keep) {
        const int k = numbers[page[u] - keep];
        if (k >= 0) *entry[u] = targets[k];
        else bad_page = true;
      }
    }
  }
  if (bad_page) atomicExch(a.status, kErrBadBlockTable);
}

__device__ __forceinline__ int wrong_length(const hs_compact_pages_t& a, int first, int stride) {
  int wrong = 0;
  for (int i = first; i < a.n_rows; i += stride) wrong |= a.ctx_len[i] < 0 || a.ctx_len[i] > row_tokens(a.max_pages_per_seq);
  return wrong;
}

// All of it in one block, bits and lists in shared memory.
__global__ void __launch_bounds__(SP_THREADS, 1) compact_small_kernel(const hs_compact_pages_t a) {
  extern __shared__ int smem[];
  __shared__ unsigned long long warp_sums[32];
  __shared__ unsigned bits[(SP_SMALL_PAGES + 31) / 32];
  const int tid = threadIdx.x;
  int *targets = smem, *numbers = smem + SP_SMALL_PAGES, *sources = smem + 2 * SP_SMALL_PAGES;
  for (int w = tid; w < (SP_SMALL_PAGES + 31) / 32; w += SP_THREADS) bits[w] = 0;
  griddep_wait();
  const int free_count = *a.free_count;
  const int wrong = __syncthreads_or(wrong_length(a, tid, SP_THREADS));
  mark_free(a, free_count, bits, tid, SP_THREADS);
  __syncthreads();
  const unsigned long long end = number_pages(a, [&](int w) { return bits[w]; }, 0, (a.num_pages + 31) / 32, 0, warp_sums, targets, numbers, sources);
  __syncthreads();
  move_pages(a, compaction_of(a, end, wrong), free_count, targets, numbers, sources, tid, SP_THREADS);
}

__global__ void __launch_bounds__(SP_THREADS, 1) compact_mark_kernel(const hs_compact_pages_t a) {
  griddep_wait();
  const int first = int(blockIdx.x) * SP_THREADS + threadIdx.x;
  mark_free(a, *a.free_count, page_bits(a.workspace), first, int(gridDim.x) * SP_THREADS);
  if (first == 0) plan_of(a)->wrong = 0;
}

// Numbers the pages: a block its share of the words, behind the sums of all words in front of it.
__global__ void __launch_bounds__(SP_THREADS, 1) compact_number_kernel(const hs_compact_pages_t a) {
  __shared__ unsigned long long warp_sums[32];
  griddep_wait();
  const int tid = threadIdx.x, n_words = (a.num_pages + 31) / 32, keep = a.n_keep;
  const unsigned* bits = page_bits(a.workspace);
  const int per_block = (n_words + int(gridDim.x) - 1) / int(gridDim.x), b0 = min(int(blockIdx.x) * per_block, n_words), b1 = min(b0 + per_block, n_words);
  // (a word in front is below the bound, or from it up, or the one that has it: counts() of number_pages)
  unsigned long long mine = 0, before = 0;
  for (int w = tid; w < b0; w += SP_THREADS) {
    const unsigned free = __ldcg(bits + w), low = keep <= w * 32 ? 0u : keep >= w * 32 + 32 ? ~0u : (1u << (keep - w * 32)) - 1u;
    mine += (static_cast<unsigned long long>(__popc(free & low)) << 32) + __popc(~free & ~low);          // (no word in front is the pool's last)
  }
  block_scan(mine, warp_sums, before);
  __syncthreads();                                       // (warp_sums)
  const unsigned long long end =
      number_pages(a, [&](int w) { return __ldcg(bits + w); }, b0, b1, before, warp_sums, targets_of(a), numbers_of(a), sources_of(a));
  Compaction* plan = plan_of(a);
  if (int(blockIdx.x) == (n_words - 1) / per_block && tid == 0) {
    const Compaction c = compaction_of(a, end, 0);
    plan->moves = c.moves;
    plan->low = c.low;
    plan->free_pages = c.free_pages;
  }
  if (wrong_length(a, int(blockIdx.x) * SP_THREADS + tid, int(gridDim.x) * SP_THREADS)) atomicExch(&plan->wrong, 1);
}

__global__ void __launch_bounds__(SP_THREADS, 1) compact_move_kernel(const hs_compact_pages_t a) {
  griddep_wait();
  const int first = int(blockIdx.x) * SP_THREADS + threadIdx.x, stride = int(gridDim.x) * SP_THREADS;
  unsigned* bits = page_bits(a.workspace);
  for (int w = first; w < (a.num_pages + 31) / 32; w += stride) bits[w] = 0;           // ready for the next call
  move_pages(a, *plan_of(a), *a.free_count, targets_of(a), numbers_of(a), sources_of(a), first, stride);
}

int grid_for(int64_t work, int64_t per_block, int sm_budget) { return int(std::max<int64_t>(1, std::min<int64_t>((work + per_block - 1) / per_block, sm_budget))); }

}  // namespace

cudaError_t shared_pages_set_attributes() {
  cudaError_t e = set_kernel_smem(fork_pages_kernel, std::max(SP_FORK_SMEM, kMinSmemBytes));
  if (e == cudaSuccess) e = set_kernel_smem(copy_pages_kernel, kMinSmemBytes);
  if (e == cudaSuccess) e = set_kernel_smem(compact_small_kernel, std::max(SP_SMALL_SMEM, kMinSmemBytes));
  if (e == cudaSuccess) e = set_kernel_smem(compact_mark_kernel, kMinSmemBytes);
  if (e == cudaSuccess) e = set_kernel_smem(compact_number_kernel, kMinSmemBytes);
  return e == cudaSuccess ? set_kernel_smem(compact_move_kernel, kMinSmemBytes) : e;
}

cudaError_t launch_fork_pages(const hs_fork_pages_t& a, int sm_budget, cudaStream_t stream) {
  const int smem = std::max(a.n_rows * (6 * 4 + SP_COLUMNS * 4), kMinSmemBytes);
  return launch_step_kernel(fork_pages_kernel, grid_for(a.max_pages_per_seq, SP_COLUMNS, sm_budget), SP_THREADS, smem, stream, true, a);
}

cudaError_t launch_copy_pages(const hs_copy_pages_t& a, int sm_budget, cudaStream_t stream) {
  const int64_t heads = int64_t(a.n_copies) * a.n_layers * 2 * a.n_kv_heads;
  return launch_step_kernel(copy_pages_kernel, grid_for(heads, 1, sm_budget), CP_THREADS, kMinSmemBytes, stream, true, a);
}

cudaError_t launch_compact_pages(const hs_compact_pages_t& a, int sm_budget, cudaStream_t stream) {
  // One launch of one block, or three of many: 1,000 pages with 1,024 entries 5.3 us for 8 to 12, 4,000 with 7,680 8.6 for 9 to 12, 8,000 with 9,216 10.9 for 9.7.
  const int64_t all_entries = int64_t(a.n_rows) * ((a.max_pages_per_seq + 31) / 32 * 32);
  if (a.num_pages <= SP_SMALL_PAGES && a.num_pages + all_entries <= SP_SMALL_WORK && a.max_copies <= SP_SMALL_PAGES)
    return launch_step_kernel(compact_small_kernel, 1, SP_THREADS, std::max(SP_SMALL_SMEM, kMinSmemBytes), stream, true, a);
  cudaError_t e = launch_step_kernel(compact_mark_kernel, grid_for(a.num_pages, SP_THREADS, sm_budget), SP_THREADS, kMinSmemBytes, stream, true, a);
  if (e == cudaSuccess) e = launch_step_kernel(compact_number_kernel, grid_for(a.num_pages, 32 * 64, sm_budget), SP_THREADS, kMinSmemBytes, stream, true, a);
  if (e != cudaSuccess) return e;
  const int64_t entries = std::max<int64_t>(int64_t(a.n_rows) * ((a.max_pages_per_seq + 31) / 32 * 32), a.num_pages);
  return launch_step_kernel(compact_move_kernel, grid_for(entries, SP_THREADS, sm_budget), SP_THREADS, kMinSmemBytes, stream, true, a);
}

}  // namespace hs
