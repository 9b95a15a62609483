// C ABI of the 4-bit cache (pagedattn_q4.h).
#include "pa_q_api.h"
#include "pagedattn_q4.h"

extern "C" {

int pa_q4_tile_bytes(int32_t head_dim, size_t* bytes) {
  if (bytes == nullptr) return PA_EINVAL;
  if (head_dim != 64 && head_dim != 128) return PA_ENOTSUP;
  *bytes = (size_t)pa::q4_tile_bytes(head_dim);
  return PA_OK;
}

int pa_kv_append_q4(const void* k_new, const void* v_new, const int32_t* block_table, const int32_t* context_lens,
                    const int32_t* query_start_loc, void* k_pages, void* v_pages, const pa_dims_t* dims, hipStream_t stream) {
  return pa::rows_call(k_new, v_new, {k_pages, v_pages, nullptr, block_table, context_lens, query_start_loc}, false, pa::kQRowsGroup,
                       dims, stream, pa::launch_q4_append);
}

int pa_kv_read_q4(const void* k_pages, const void* v_pages, const int32_t* block_table, const int32_t* context_lens,
                  const int32_t* query_start_loc, void* k_out, void* v_out, const pa_dims_t* dims, hipStream_t stream) {
  return pa::rows_call(k_out, v_out, {k_pages, v_pages, nullptr, block_table, context_lens, query_start_loc}, false, pa::kQRowsGroup,
                       dims, stream, pa::launch_q4_read);
}

int pa_workspace_size_q4(const pa_dims_t* dims, size_t* bytes) {
  return pa::workspace_bytes_of<pa::q4::Format>(dims, bytes);
}

int paged_attn_q4(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                  const int32_t* context_lens, float scale, void* out, const pa_dims_t* dims, void* workspace,
                  size_t workspace_bytes, hipStream_t stream, const pa_timing_t* timing) {
  return pa::attend<pa::q4::Format>(q, {k_pages, v_pages, nullptr, block_table, context_lens, nullptr}, false, scale, out, dims,
                                    workspace, workspace_bytes, stream, timing, false);
}

int paged_attn_varlen_q4(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                         const int32_t* context_lens, const int32_t* query_start_loc, float scale, void* out,
                         const pa_dims_t* dims, void* workspace, size_t workspace_bytes, hipStream_t stream,
                         const pa_timing_t* timing) {
  return pa::attend<pa::q4::Format>(q, {k_pages, v_pages, nullptr, block_table, context_lens, query_start_loc}, false, scale, out, dims,
                                    workspace, workspace_bytes, stream, timing, true);
}

}  // extern "C"
