// C entry points of horizonserve_device.h and horizonserve_beams.h: checks of the arguments, tensor maps, launches.
#include <mutex>

#include "device_ops.h"
#include "hs_internal.h"

namespace hs {
namespace {

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// What a call needs to know of the current device; set up once per device.
struct Device {
  bool ready = false;
  int sm_count = 0;
};
std::mutex g_mutex;
Device g_device[64];
EncodeTiledFn g_encode = nullptr;

hs_status_t set_up(int dev, Device& d) {
  int sm = 0, major = 0;
  cudaError_t e = cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  if (e != cudaSuccess) return report_cuda_error("device attributes", e);
  if (major != 10) return report_cuda_error("the device is not compute capability 10.x", cudaErrorInvalidDevice);
  if (!g_encode) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
    if (e != cudaSuccess || q != cudaDriverEntryPointSuccess) return report_cuda_error("cuTensorMapEncodeTiled", e != cudaSuccess ? e : cudaErrorNotSupported);
    g_encode = reinterpret_cast<EncodeTiledFn>(fn);
  }
  if ((e = step_tables_set_attributes()) != cudaSuccess) return report_cuda_error("page table attributes", e);
  if ((e = rope_cache_set_attributes()) != cudaSuccess) return report_cuda_error("rope attributes", e);
  if ((e = paged_decode_set_attributes()) != cudaSuccess) return report_cuda_error("paged decode attributes", e);
  if ((e = paged_chunk_set_attributes()) != cudaSuccess) return report_cuda_error("paged chunk attributes", e);
  if ((e = token_logprobs_set_attributes()) != cudaSuccess) return report_cuda_error("log probability attributes", e);
  if ((e = beam_select_set_attributes()) != cudaSuccess) return report_cuda_error("beam selection attributes", e);
  if ((e = shared_pages_set_attributes()) != cudaSuccess) return report_cuda_error("shared page attributes", e);
  if ((e = shared_attention_set_attributes()) != cudaSuccess) return report_cuda_error("shared attention attributes", e);
  d.sm_count = sm;
  d.ready = true;
  return HS_OK;
}

// The current device, and whether sm_budget is one of its budgets.
hs_status_t enter(int sm_budget, const Device** out) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda_error("cudaGetDevice", e);
  if (dev < 0 || dev >= 64) return report_cuda_error("device ordinal", cudaErrorInvalidDevice);
  std::lock_guard<std::mutex> lock(g_mutex);
  Device& d = g_device[dev];
  if (!d.ready) {
    const hs_status_t st = set_up(dev, d);
    if (st != HS_OK) return st;
  }
  if (sm_budget < 1 || sm_budget > d.sm_count) return HS_ERR_INVALID_BUDGET;
  *out = &d;
  return HS_OK;
}

hs_status_t launched(const char* where, cudaError_t e) { return e == cudaSuccess ? HS_OK : report_cuda_error(where, e); }

// Rows of `cols` 16-bit elements, `stride` elements apart; box of 64 columns x box_rows, 128-byte swizzle.
bool encode_rows(CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows) {
  cuuint64_t dims[2] = {cols, rows};
  cuuint64_t strides[1] = {stride * 2};
  cuuint32_t box[2] = {64, box_rows};
  cuuint32_t estr[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Sequences of heads of `dim` 16-bit elements, sequences `stride` elements apart; box of 64 columns x box_heads x box_seqs, 128-byte swizzle.
bool encode_heads(CUtensorMap* m, const void* base, uint64_t seqs, uint64_t heads, uint64_t dim, uint64_t stride, uint32_t box_seqs, uint32_t box_heads) {
  cuuint64_t dims[3] = {dim, heads, seqs};
  cuuint64_t strides[2] = {dim * 2, stride * 2};
  cuuint32_t box[3] = {64, box_heads, box_seqs};
  cuuint32_t estr[3] = {1, 1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool tables_shape_ok(int n_seqs, int max_pages) { return n_seqs <= HS_DEVICE_MAX_SEQS && int64_t(n_seqs) * max_pages <= (int64_t(1) << 27); }
bool workspace_ok(const void* w) { return w && aligned(w, 256); }

}  // namespace
}  // namespace hs

using namespace hs;

extern "C" {

hs_status_t hs_op_step_tables(const hs_step_tables_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_seqs < 1 || a->max_pages_per_seq < 1 || a->num_pages < 1 || a->max_tokens < 1) return HS_ERR_INVALID_ARG;
  if (!a->ctx_len || !a->q_len || !a->free_list || !a->free_count || !a->block_tables || !a->kv_len || !a->tok_begin || !a->tok_seq || !a->tok_pos ||
      !a->tok_slot || !a->free_count_out || !a->status || !workspace_ok(a->workspace))
    return HS_ERR_INVALID_ARG;
  if (!tables_shape_ok(a->n_seqs, a->max_pages_per_seq) || a->num_pages >= (1 << 27)) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("step tables", launch_step_tables(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_release_pages(const hs_release_pages_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_seqs < 1 || a->max_pages_per_seq < 1 || a->num_pages < 1) return HS_ERR_INVALID_ARG;
  if (!a->done || !a->ctx_len || !a->block_tables || !a->free_list || !a->free_count || !a->status || !workspace_ok(a->workspace)) return HS_ERR_INVALID_ARG;
  if (!tables_shape_ok(a->n_seqs, a->max_pages_per_seq) || a->num_pages >= (1 << 27)) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("release pages", launch_release_pages(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_rope_table(const hs_rope_table_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || !a->table || a->max_position < 1 || !aligned(a->table, 16)) return HS_ERR_INVALID_ARG;
  if (a->rotary_dim < 16 || a->rotary_dim > 256 || a->rotary_dim % 16 != 0) return HS_ERR_UNSUPPORTED_SHAPE;
  if (a->scaling < HS_ROPE_PLAIN || a->scaling > HS_ROPE_BY_PARTS || !(a->base > 0.0) || !(a->magnitude > 0.0)) return HS_ERR_INVALID_ARG;
  if (a->scaling != HS_ROPE_PLAIN && !(a->factor > 0.0)) return HS_ERR_INVALID_ARG;
  if (a->scaling == HS_ROPE_BY_PARTS && (a->trained_positions < 1 || !(a->turns_fast > a->turns_slow))) return HS_ERR_INVALID_ARG;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("rope table", launch_rope_table(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_rope_cache(const hs_rope_cache_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_tokens < 1 || a->n_q_heads < 1 || a->n_kv_heads < 1 || a->max_position < 1) return HS_ERR_INVALID_ARG;
  if (!a->q || !a->k || !a->v || !a->tok_pos || !a->tok_slot || !a->table || !a->q_out || !a->kv_pool || !a->status) return HS_ERR_INVALID_ARG;
  if (a->n_layers < 1 || a->layer < 0 || a->layer >= a->n_layers || a->num_pages < 1) return HS_ERR_INVALID_ARG;
  if (a->src_type < HS_TYPE_F32 || a->src_type > HS_TYPE_F16 || (a->cache_type != HS_TYPE_BF16 && a->cache_type != HS_TYPE_F16)) return HS_ERR_INVALID_ARG;
  if (a->head_dim < 16 || a->head_dim > 256 || a->head_dim % 16 != 0 || a->rotary_dim < 16 || a->rotary_dim > a->head_dim || a->rotary_dim % 16 != 0 ||
      a->n_q_heads > 1024 || a->n_kv_heads > 1024 || a->num_pages >= (1 << 27))
    return HS_ERR_UNSUPPORTED_SHAPE;
  const int64_t q_row = int64_t(a->n_q_heads) * a->head_dim, kv_row = int64_t(a->n_kv_heads) * a->head_dim;
  const int piece = a->src_type == HS_TYPE_F32 ? 4 : 8;
  if (a->q_stride < q_row || a->k_stride < kv_row || a->v_stride < kv_row || a->q_out_stride < q_row) return HS_ERR_INVALID_ARG;
  if (a->q_stride % piece || a->k_stride % piece || a->v_stride % piece || a->q_out_stride % 8 || !aligned(a->q, 16) || !aligned(a->k, 16) ||
      !aligned(a->v, 16) || !aligned(a->q_out, 16) || !aligned(a->table, 16) || !aligned(a->kv_pool, 256))
    return HS_ERR_INVALID_ARG;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("rope and cache write", launch_rope_cache(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_paged_attention(const hs_paged_attention_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_seqs < 1 || a->n_tokens < 1 || a->max_q_len < 1 || a->n_q_heads < 1 || a->n_kv_heads < 1) return HS_ERR_INVALID_ARG;
  if (!a->q || !a->kv_pool || !a->block_tables || !a->kv_len || !a->o || !a->status || !workspace_ok(a->workspace)) return HS_ERR_INVALID_ARG;
  if (a->n_layers < 1 || a->layer < 0 || a->layer >= a->n_layers || a->num_pages < 1 || a->max_pages_per_seq < 1) return HS_ERR_INVALID_ARG;
  if (a->type != HS_TYPE_BF16 && a->type != HS_TYPE_F16) return HS_ERR_INVALID_ARG;
  if (!a->tok_begin && (a->max_q_len != 1 || a->n_tokens < a->n_seqs)) return HS_ERR_INVALID_ARG;
  if (!(a->cap >= 0.f && a->cap < 1e30f) || !(a->scale > -1e30f && a->scale < 1e30f) || a->window < 0) return HS_ERR_INVALID_ARG;
  if ((a->head_dim != 64 && a->head_dim != 128) || a->n_q_heads % a->n_kv_heads != 0 || a->n_q_heads > 1024) return HS_ERR_UNSUPPORTED_SHAPE;
  const int64_t q_row = int64_t(a->n_q_heads) * a->head_dim;
  if (a->q_stride < q_row || a->o_stride < q_row || a->q_stride % 8 || a->o_stride % 8) return HS_ERR_INVALID_ARG;
  if (!aligned(a->q, 16) || !aligned(a->o, 16) || !aligned(a->kv_pool, 256)) return HS_ERR_INVALID_ARG;
  // (rows of the pool are counted in 32 bits, and so are the keys of a block table row)
  const int64_t rows = int64_t(a->n_layers) * 2 * a->num_pages * a->n_kv_heads * kPage;
  if (!tables_shape_ok(a->n_seqs, a->max_pages_per_seq) || rows >= (int64_t(1) << 31)) return HS_ERR_UNSUPPORTED_SHAPE;
  // (so are the pages of all sequences and groups of heads one after the other, and the tiles of a chunk's tokens)
  if (int64_t(a->n_seqs) * a->max_pages_per_seq * a->n_q_heads >= (int64_t(1) << 31) || int64_t(a->n_tokens) * a->n_q_heads >= (int64_t(1) << 31)) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  CUtensorMap tm_kv, tm_q;
  if (a->max_q_len == 1) {
    if (!encode_kv_pages(g_encode, &tm_kv, a->kv_pool, a->n_layers, a->num_pages, a->n_kv_heads, a->head_dim))
      return report_cuda_error("tensor map", cudaErrorInvalidValue);
    return launched("paged decode attention", launch_paged_decode(*a, tm_kv, d->sm_count, sm_budget, stream));
  }
  if (!encode_rows(&tm_kv, a->kv_pool, rows, a->head_dim, a->head_dim, kPage) ||
      !encode_rows(&tm_q, a->q, a->n_tokens, q_row, a->q_stride, paged_chunk_tile_tokens(a->n_q_heads, a->n_kv_heads)))
    return report_cuda_error("tensor map", cudaErrorInvalidValue);
  return launched("paged chunk attention", launch_paged_chunk(*a, tm_kv, tm_q, d->sm_count, sm_budget, stream));
}

hs_status_t hs_op_token_logprobs(const hs_token_logprobs_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_rows < 1 || a->vocab < 1 || a->row_stride < a->vocab) return HS_ERR_INVALID_ARG;
  if (!a->logits || !a->targets || !a->logprob || !a->status || !workspace_ok(a->workspace)) return HS_ERR_INVALID_ARG;
  if (a->type < HS_TYPE_F32 || a->type > HS_TYPE_F16 || !aligned(a->logits, a->type == HS_TYPE_F32 ? 4 : 2)) return HS_ERR_INVALID_ARG;
  if (a->n_top < 0 || (a->n_top > 0 && (!a->top_ids || !a->top_logprobs)) || !(a->scale > 0.f && a->scale < 1e30f)) return HS_ERR_INVALID_ARG;
  if (a->n_top > HS_MAX_ALTERNATIVES || a->n_top > a->vocab || a->vocab >= (1 << 30)) return HS_ERR_UNSUPPORTED_SHAPE;
  if (int64_t(a->n_rows) * (a->vocab / 1024 + 2) >= (int64_t(1) << 31)) return HS_ERR_UNSUPPORTED_SHAPE;        // (the kernel counts in units of 1024)
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("token log probabilities", launch_token_logprobs(*a, d->sm_count, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_beam_select(const hs_beam_select_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_requests < 1 || a->n_beams < 1 || a->vocab < 1 || a->n_out < 1 || a->row_stride < a->vocab) return HS_ERR_INVALID_ARG;
  if (!a->logits || !a->scores || !a->out_score || !a->out_parent || !a->out_token || !a->status || !workspace_ok(a->workspace)) return HS_ERR_INVALID_ARG;
  if (a->type < HS_TYPE_F32 || a->type > HS_TYPE_F16 || !aligned(a->logits, a->type == HS_TYPE_F32 ? 4 : 2)) return HS_ERR_INVALID_ARG;
  if (!(a->scale > 0.f && a->scale < 1e30f)) return HS_ERR_INVALID_ARG;
  if (a->n_requests > HS_DEVICE_MAX_SEQS || a->n_beams > HS_MAX_BEAMS || a->n_out > HS_MAX_BEAMS || a->vocab >= (1 << 30)) return HS_ERR_UNSUPPORTED_SHAPE;
  if (int64_t(a->n_requests) * a->n_beams > 65536) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("beam selection", launch_beam_select(*a, d->sm_count, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_fork_pages(const hs_fork_pages_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_rows < 1 || a->max_pages_per_seq < 1 || a->num_pages < 1) return HS_ERR_INVALID_ARG;
  if (!a->parent || !a->ctx_len || !a->block_tables || !a->shares || !a->free_list || !a->free_count || !a->copy_src || !a->copy_dst || !a->copy_len ||
      !a->status || !workspace_ok(a->workspace))
    return HS_ERR_INVALID_ARG;
  if (!tables_shape_ok(a->n_rows, a->max_pages_per_seq) || a->num_pages > HS_BEAMS_MAX_PAGES) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("fork pages", launch_fork_pages(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_copy_pages(const hs_copy_pages_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_copies < 1 || a->n_layers < 1 || a->num_pages < 1 || a->n_kv_heads < 1 || a->head_dim < 1) return HS_ERR_INVALID_ARG;
  if (!a->src || !a->dst || !a->kv_pool || !a->status || !aligned(a->kv_pool, 256)) return HS_ERR_INVALID_ARG;
  if (a->type != HS_TYPE_BF16 && a->type != HS_TYPE_F16) return HS_ERR_INVALID_ARG;
  if (a->head_dim % 8 != 0 || a->head_dim > 256 || a->n_kv_heads > 1024 || a->num_pages >= (1 << 27) || a->n_copies > HS_COMPACT_MAX_PAGES) return HS_ERR_UNSUPPORTED_SHAPE;
  if (int64_t(a->n_layers) * 2 * a->n_kv_heads >= (int64_t(1) << 31) / a->n_copies) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("copy pages", launch_copy_pages(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_compact_pages(const hs_compact_pages_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_rows < 1 || a->max_pages_per_seq < 1 || a->num_pages < 1 || a->n_keep < 0 || a->n_keep > a->num_pages || a->max_copies < 0) return HS_ERR_INVALID_ARG;
  if (!a->ctx_len || !a->block_tables || !a->shares || !a->free_list || !a->free_count || (a->max_copies > 0 && (!a->copy_src || !a->copy_dst)) || !a->status ||
      !workspace_ok(a->workspace))
    return HS_ERR_INVALID_ARG;
  if (!tables_shape_ok(a->n_rows, a->max_pages_per_seq) || a->num_pages > HS_COMPACT_MAX_PAGES) return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  return launched("compact pages", launch_compact_pages(*a, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

hs_status_t hs_op_shared_attention(const hs_shared_attention_t* a, int32_t sm_budget, void* cuda_stream) {
  if (!a || a->n_seqs < 1 || a->n_groups < 1 || a->n_groups > a->n_seqs || a->n_q_heads < 1 || a->n_kv_heads < 1) return HS_ERR_INVALID_ARG;
  if (!a->q || !a->kv_pool || !a->block_tables || !a->kv_len || !a->group_begin || !a->shared_len || !a->o || !a->status || !workspace_ok(a->workspace))
    return HS_ERR_INVALID_ARG;
  if (a->n_layers < 1 || a->layer < 0 || a->layer >= a->n_layers || a->num_pages < 1 || a->max_pages_per_seq < 1) return HS_ERR_INVALID_ARG;
  if (a->type != HS_TYPE_BF16 && a->type != HS_TYPE_F16) return HS_ERR_INVALID_ARG;
  if (!(a->cap >= 0.f && a->cap < 1e30f) || !(a->scale > -1e30f && a->scale < 1e30f)) return HS_ERR_INVALID_ARG;
  if ((a->head_dim != 64 && a->head_dim != 128) || a->n_q_heads % a->n_kv_heads != 0 || a->n_q_heads > 1024) return HS_ERR_UNSUPPORTED_SHAPE;
  const int64_t q_row = int64_t(a->n_q_heads) * a->head_dim;
  if (a->q_stride < q_row || a->o_stride < q_row || a->q_stride % 8 || a->o_stride % 8) return HS_ERR_INVALID_ARG;
  if (!aligned(a->q, 16) || !aligned(a->o, 16) || !aligned(a->kv_pool, 256)) return HS_ERR_INVALID_ARG;
  const int64_t rows = int64_t(a->n_layers) * 2 * a->num_pages * a->n_kv_heads * kPage;
  if (!tables_shape_ok(a->n_seqs, a->max_pages_per_seq) || rows >= (int64_t(1) << 31)) return HS_ERR_UNSUPPORTED_SHAPE;
  // (the blocks of all tiles one after the other are counted in 32 bits, and so are the keys of a tile)
  if (a->n_seqs > HS_SHARED_MAX_SEQS || int64_t(a->n_seqs) * a->max_pages_per_seq > (int64_t(1) << 26) || int64_t(a->n_seqs) * a->max_pages_per_seq * a->n_q_heads >= (int64_t(1) << 30))
    return HS_ERR_UNSUPPORTED_SHAPE;
  const Device* d = nullptr;
  const hs_status_t st = enter(sm_budget, &d);
  if (st != HS_OK) return st;
  CUtensorMap tm_q;
  const SharedTile tile = shared_attention_tile(*a);
  if (!encode_heads(&tm_q, a->q, a->n_seqs, a->n_q_heads, a->head_dim, a->q_stride, tile.seqs, tile.heads)) return report_cuda_error("tensor map", cudaErrorInvalidValue);
  return launched("shared attention", launch_shared_attention(*a, tm_q, d->sm_count, sm_budget, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
