// Page allocation and per-token metadata of a step from lengths that are on the device, and the return of finished requests' pages.
//
//   pages of request s   owned_s = ceil(ctx_s / 16),  new_s = ceil((ctx_s + q_s) / 16) - owned_s
//   two running sums     T_s = sum of q, P_s = sum of new pages over the requests in front of s
//   a new page           entry owned_s + i of row s = free_list[free_count - 1 - P_s - i]
//   a token              t in [T_s, T_s + q_s): position ctx_s + t - T_s, slot = page * 16 + position % 16
//
// Everything follows from the two sums, so every block forms them for itself in shared memory (4096 requests are four a thread)
// and no block waits for another: a token finds its request by bisection, and the id of a page that this step allocates straight
// from the free list.  A few microseconds of latency is all there is -- 3.8 us for 64
// requests, 4.8 for 1000 with 12402 tokens --: the launch, one round trip for the lengths, the scan, one for the ids.  Pages go back
// in one pass over their entries: 4.2 us for seven, 4.8 for 64 requests' 16384, 6.9 for 256000.
#include <algorithm>

#include "device_ops.h"
#include "ptx.cuh"

namespace hs {
namespace {

constexpr int TB_THREADS = 1024, TB_PER_THREAD = HS_DEVICE_MAX_SEQS / TB_THREADS;
static_assert(2 * (HS_DEVICE_MAX_SEQS + 1) * 4 <= kMinSmemBytes, "both sums in shared memory");

// Exclusive running sums over the block's threads of a pair of counts below 2^31, packed in 64 bits; `total` is the same in every thread.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* warp_sums, unsigned long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += x;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  unsigned long long w = warp_sums[lane];               // (32 warps)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += x;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const unsigned long long before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return (warp > 0 ? before : 0ull) + inc - v;
}

// The last s in 0 .. n - 1 with begin[s] <= x; begin has n + 1 entries and begin[n] > x.
__device__ __forceinline__ int find(const int* begin, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ bool last_block(int* done) {
  __shared__ int last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(done, 1) == int(gridDim.x) - 1;
    if (last) *done = 0;                                 // ready for the next call
    __threadfence();
  }
  __syncthreads();
  return last != 0;
}

__global__ void __launch_bounds__(TB_THREADS, 1) step_tables_kernel(const hs_step_tables_t a, const int in_place) {
  extern __shared__ int sums[];
  __shared__ unsigned long long warp_sums[32];
  griddep_wait();
  const int n = a.n_seqs, tid = threadIdx.x;
  int* tok_begin = sums;
  int* page_begin = sums + n + 1;

  const int free_count = *a.free_count;
  int ctx[TB_PER_THREAD], q[TB_PER_THREAD], wrong = 0;
  unsigned long long mine = 0;
  const int most = row_tokens(a.max_pages_per_seq);
#pragma unroll
  for (int i = 0; i < TB_PER_THREAD; ++i) {
    const int s = tid * TB_PER_THREAD + i;
    ctx[i] = s < n ? a.ctx_len[s] : 0;
    q[i] = s < n ? a.q_len[s] : 0;
    if (ctx[i] < 0 || q[i] < 0 || ctx[i] > most || q[i] > most - ctx[i]) {
      wrong = 1;
      q[i] = 0;
      ctx[i] = 0;
    }
    mine += (static_cast<unsigned long long>(((ctx[i] + q[i] + 15) >> 4) - ((ctx[i] + 15) >> 4)) << 32) + unsigned(q[i]);
  }
  unsigned long long total;
  unsigned long long at = block_scan(mine, warp_sums, total);
#pragma unroll
  for (int i = 0; i < TB_PER_THREAD; ++i) {
    const int s = tid * TB_PER_THREAD + i;
    if (s < n) {
      tok_begin[s] = int(unsigned(at));
      page_begin[s] = int(at >> 32);
    }
    at += (static_cast<unsigned long long>(((ctx[i] + q[i] + 15) >> 4) - ((ctx[i] + 15) >> 4)) << 32) + unsigned(q[i]);
  }
  int n_tokens = int(unsigned(total)), n_new = int(total >> 32);
  if (tid == 0) {
    tok_begin[n] = n_tokens;
    page_begin[n] = n_new;
  }
  wrong = __syncthreads_or(wrong);                       // (the sums are in shared memory for everybody, too)
  int error = 0;
  if (wrong || unsigned(n_tokens) > unsigned(a.max_tokens) || free_count < 0 || free_count > a.num_pages) error = kErrInvalidArg;
  else if (n_new > free_count) error = kErrOutOfPages;
  if (error) n_tokens = n_new = 0;

  const int stride = gridDim.x * TB_THREADS, first = blockIdx.x * TB_THREADS + tid;
  int bad_page = 0;
  // (a capacity just below 2^31 is one that the last step of t passes)
  for (unsigned u = first; u < unsigned(a.max_tokens); u += stride) {
    const int t = int(u);
    int seq = -1, pos = -1, slot = -1;
    if (t < n_tokens) {
      seq = find(tok_begin, n, t);
      const int c = a.ctx_len[seq], owned = (c + 15) >> 4;
      pos = c + (t - tok_begin[seq]);
      const int i = (pos >> 4) - owned;                  // of the pages this step allocates, or negative
      const int page = i >= 0 ? a.free_list[free_count - 1 - page_begin[seq] - i] : a.block_tables[size_t(seq) * a.max_pages_per_seq + (pos >> 4)];
      if (page >= 0 && page < a.num_pages) slot = page * 16 + (pos & 15);
      else bad_page = 1;
    }
    a.tok_seq[t] = seq;
    a.tok_pos[t] = pos;
    a.tok_slot[t] = slot;
  }
  for (int i = first; i < n_new; i += stride) {
    const int s = find(page_begin, n, i);
    a.block_tables[size_t(s) * a.max_pages_per_seq + ((a.ctx_len[s] + 15) >> 4) + i - page_begin[s]] = a.free_list[free_count - 1 - i];
  }
  if (bad_page) atomicExch(a.status, kErrBadBlockTable);
  if (error && first == 0) atomicExch(a.status, error);

  // what may lie where another block still reads is written by the last block; the rest at once, by the first
  if (in_place ? !last_block(reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsTables)) : blockIdx.x != 0) return;
#pragma unroll
  for (int i = 0; i < TB_PER_THREAD; ++i) {
    const int s = tid * TB_PER_THREAD + i;
    if (s >= n) continue;
    a.kv_len[s] = error ? a.ctx_len[s] : ctx[i] + q[i];
    a.tok_begin[s] = error ? 0 : tok_begin[s];
  }
  if (tid == 0) {
    a.tok_begin[n] = n_tokens;
    *a.free_count_out = free_count - n_new;
  }
}

__global__ void __launch_bounds__(TB_THREADS, 1) release_pages_kernel(const hs_release_pages_t a) {
  extern __shared__ int sums[];
  __shared__ unsigned long long warp_sums[32];
  griddep_wait();
  const int n = a.n_seqs, tid = threadIdx.x;
  int* page_begin = sums;
  const int free_count = *a.free_count;
  int pages[TB_PER_THREAD], wrong = 0;
  bool done[TB_PER_THREAD];
  unsigned long long mine = 0;
#pragma unroll
  for (int i = 0; i < TB_PER_THREAD; ++i) {
    const int s = tid * TB_PER_THREAD + i;
    done[i] = s < n && a.done[s] != 0;
    const int ctx = done[i] ? a.ctx_len[s] : 0;
    if (ctx < 0 || ctx > row_tokens(a.max_pages_per_seq)) wrong = 1;
    pages[i] = wrong ? 0 : (ctx + 15) >> 4;
    mine += unsigned(pages[i]);
  }
  unsigned long long total;
  int at = int(block_scan(mine, warp_sums, total));
#pragma unroll
  for (int i = 0; i < TB_PER_THREAD; ++i) {
    const int s = tid * TB_PER_THREAD + i;
    if (s < n) page_begin[s] = at;
    at += pages[i];
  }
  const int n_back = int(total);
  if (tid == 0) page_begin[n] = n_back;
  wrong = __syncthreads_or(wrong);
  const bool ok = !wrong && free_count >= 0 && n_back <= a.num_pages - free_count;
  // What lies behind the stack's top belongs to nobody: the pages go there first, and are on the stack when the last block moves its top.  If one of them is
  // outside the pool it does not, and puts the block tables' entries back from there instead.
  int* words = reinterpret_cast<int*>(static_cast<char*>(a.workspace) + kWsTables);
  auto entry_of = [&](int i) {                            // of the i-th page that goes back: a request's last page first
    const int s = find(page_begin, n, i);
    return a.block_tables + size_t(s) * a.max_pages_per_seq + (page_begin[s + 1] - 1 - i);
  };
  bool bad_page = false;
  if (ok) {
    for (int i = blockIdx.x * TB_THREADS + tid; i < n_back; i += gridDim.x * TB_THREADS) {
      int32_t* entry = entry_of(i);
      const int page = *entry;
      bad_page |= page < 0 || page >= a.num_pages;
      a.free_list[free_count + i] = page;
      *entry = -1;
    }
  }
  if (bad_page) atomicExch(words + 1, 1);
  if (!last_block(words)) return;
  if (!ok) {
    if (tid == 0) atomicExch(a.status, kErrInvalidArg);
    return;
  }
  if (__ldcg(words + 1) != 0) {
    for (int i = tid; i < n_back; i += TB_THREADS) *entry_of(i) = __ldcg(a.free_list + free_count + i);
    __syncthreads();
    if (tid == 0) {
      words[1] = 0;                                      // ready for the next call
      atomicExch(a.status, kErrBadBlockTable);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < TB_PER_THREAD; ++i)
    if (done[i]) a.ctx_len[tid * TB_PER_THREAD + i] = 0;
  if (tid == 0) *a.free_count = free_count + n_back;
}

int tables_grid(int64_t work, int sm_budget) {
  const int64_t blocks = (work + TB_THREADS - 1) / TB_THREADS;
  return int(blocks < 1 ? 1 : blocks < sm_budget ? blocks : sm_budget);
}

}  // namespace

cudaError_t step_tables_set_attributes() {
  const cudaError_t e = set_kernel_smem(step_tables_kernel, kMinSmemBytes);
  return e != cudaSuccess ? e : set_kernel_smem(release_pages_kernel, kMinSmemBytes);
}

cudaError_t launch_step_tables(const hs_step_tables_t& a, int sm_budget, cudaStream_t stream) {
  const int in_place = a.kv_len == a.ctx_len || a.free_count_out == a.free_count;
  const int grid = tables_grid(a.max_tokens, sm_budget);
  return launch_step_kernel(step_tables_kernel, grid, TB_THREADS, kMinSmemBytes, stream, true, a, in_place);
}

cudaError_t launch_release_pages(const hs_release_pages_t& a, int sm_budget, cudaStream_t stream) {
  const int grid = tables_grid(std::min<int64_t>(int64_t(a.n_seqs) * a.max_pages_per_seq, a.num_pages), sm_budget);
  return launch_step_kernel(release_pages_kernel, grid, TB_THREADS, kMinSmemBytes, stream, true, a);
}

}  // namespace hs
