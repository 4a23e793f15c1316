// Launchers of the operators of horizonserve_device.h and horizonserve_beams.h.  Each takes the caller's description, already checked, and the device's SM
// count; it enqueues one persistent kernel of at most sm_budget blocks.
#pragma once
#include <cuda_runtime.h>

#include "../../include/horizonserve_beams.h"
#include "kernels.h"

namespace hs {

// The caller's workspace.  Control words are zero between calls; scratch holds nothing across calls.
constexpr size_t kWsTables = 0;              // two words: blocks that are done; whether one of them found a page outside the pool
constexpr size_t kWsAttnDone = 1024;         // one word per share: parts delivered of the group that begins in it
constexpr size_t kWsLogprobsDone = 4096;     // the same for logit rows
constexpr size_t kWsChunkQueue = 8192;       // work queue of the chunk attention, and blocks that have left it
constexpr size_t kWsChunkDone = 16 << 10;    // its divided items: warps' rows of parts delivered, tile by tile
constexpr size_t kWsSelectQueue = 24 << 10;  // work queue of the beam selection, and blocks that have left it
constexpr size_t kWsSelectDone = 28 << 10;   // one word per request: parts of its rows that are done
constexpr size_t kWsSharedQueue = 48 << 10;  // shared attention: one word per share, parts delivered of the item that begins in it
constexpr size_t kWsScratch = 64 << 10;
constexpr size_t kWsPageBits = HS_DEVICE_WORKSPACE_BYTES - (HS_BEAMS_MAX_PAGES / 8);   // a bit per page of the pool, zero between calls
constexpr size_t kWsScratchBytes = kWsPageBits - kWsScratch;
// Shares that the work of a split operator is cut into: one per SM of the device, never more than this.
constexpr int kMaxShares = 160;

// Tokens of a sequence whose block table row has that many pages.  Lengths, and lengths rounded up to whole pages or blocks of 64 keys, are 32-bit numbers, so
// the last 64 tokens of a row of 2^27 pages are not to be had.
__host__ __device__ inline int row_tokens(int max_pages) { return max_pages < (1 << 27) - 4 ? max_pages * HS_PAGE_SIZE : ((1 << 27) - 4) * HS_PAGE_SIZE; }

inline int share_count(int sm_count) { return sm_count < kMaxShares ? sm_count : kMaxShares; }

constexpr int kErrOutOfPages = HS_ERR_OUT_OF_PAGES, kErrBadBlockTable = HS_ERR_BAD_BLOCK_TABLE;

cudaError_t step_tables_set_attributes();
cudaError_t launch_step_tables(const hs_step_tables_t& a, int sm_budget, cudaStream_t stream);
cudaError_t launch_release_pages(const hs_release_pages_t& a, int sm_budget, cudaStream_t stream);

cudaError_t rope_cache_set_attributes();
cudaError_t launch_rope_table(const hs_rope_table_t& a, int sm_budget, cudaStream_t stream);
cudaError_t launch_rope_cache(const hs_rope_cache_t& a, int sm_budget, cudaStream_t stream);

cudaError_t paged_decode_set_attributes();
cudaError_t launch_paged_decode(const hs_paged_attention_t& a, const CUtensorMap& tm_kv_page, int sm_count, int sm_budget, cudaStream_t stream);
cudaError_t paged_chunk_set_attributes();
cudaError_t launch_paged_chunk(const hs_paged_attention_t& a, const CUtensorMap& tm_kv, const CUtensorMap& tm_q, int sm_count, int sm_budget, cudaStream_t stream);
int paged_chunk_tile_tokens(int n_q_heads, int n_kv_heads);      // token rows of tm_q's box

cudaError_t token_logprobs_set_attributes();
cudaError_t launch_token_logprobs(const hs_token_logprobs_t& a, int sm_count, int sm_budget, cudaStream_t stream);

cudaError_t beam_select_set_attributes();
cudaError_t launch_beam_select(const hs_beam_select_t& a, int sm_count, int sm_budget, cudaStream_t stream);

cudaError_t shared_pages_set_attributes();
cudaError_t launch_fork_pages(const hs_fork_pages_t& a, int sm_budget, cudaStream_t stream);
cudaError_t launch_copy_pages(const hs_copy_pages_t& a, int sm_budget, cudaStream_t stream);
cudaError_t launch_compact_pages(const hs_compact_pages_t& a, int sm_budget, cudaStream_t stream);

cudaError_t shared_attention_set_attributes();
cudaError_t launch_shared_attention(const hs_shared_attention_t& a, const CUtensorMap& tm_q, int sm_count, int sm_budget, cudaStream_t stream);
struct SharedTile {
  int heads, seqs, copies;                                       // of tm_q's box: query heads, sequences; how often a tile's rows stand in the matrix
};
SharedTile shared_attention_tile(const hs_shared_attention_t& a);

}  // namespace hs
