// C ABI of the 8-bit cache (pagedattn_q8.h).
#include "pa_q_api.h"
#include "pagedattn_q8.h"

namespace {

bool misaligned2(const void* p) { return ((uintptr_t)p & 1) != 0; }

}  // namespace

extern "C" {

int pa_kv_append_q8(const void* k_new, const void* v_new, const int32_t* block_table, const int32_t* context_lens,
                    const int32_t* query_start_loc, void* k_pages, void* v_pages, uint8_t* scales, const pa_dims_t* dims,
                    hipStream_t stream) {
  if (misaligned2(scales)) return PA_EINVAL;
  return pa::rows_call(k_new, v_new, {k_pages, v_pages, scales, block_table, context_lens, query_start_loc}, true, 16, dims, stream,
                       pa::launch_q8_append);
}

int pa_kv_read_q8(const void* k_pages, const void* v_pages, const uint8_t* scales, const int32_t* block_table,
                  const int32_t* context_lens, const int32_t* query_start_loc, void* k_out, void* v_out, const pa_dims_t* dims,
                  hipStream_t stream) {
  if (misaligned2(scales)) return PA_EINVAL;
  return pa::rows_call(k_out, v_out, {k_pages, v_pages, scales, block_table, context_lens, query_start_loc}, true, pa::kQRowsGroup,
                       dims, stream, pa::launch_q8_read);
}

int pa_workspace_size_q8(const pa_dims_t* dims, size_t* bytes) {
  return pa::workspace_bytes_of<pa::q8::Format>(dims, bytes);
}

int paged_attn_q8(const void* q, const void* k_pages, const void* v_pages, const uint8_t* scales, const int32_t* block_table,
                  const int32_t* context_lens, float scale, void* out, const pa_dims_t* dims, void* workspace,
                  size_t workspace_bytes, hipStream_t stream, const pa_timing_t* timing) {
  if (misaligned2(scales)) return PA_EINVAL;
  return pa::attend<pa::q8::Format>(q, {k_pages, v_pages, scales, block_table, context_lens, nullptr}, true, scale, out, dims,
                                    workspace, workspace_bytes, stream, timing, false);
}

int paged_attn_varlen_q8(const void* q, const void* k_pages, const void* v_pages, const uint8_t* scales,
                         const int32_t* block_table, const int32_t* context_lens, const int32_t* query_start_loc, float scale,
                         void* out, const pa_dims_t* dims, void* workspace, size_t workspace_bytes, hipStream_t stream,
                         const pa_timing_t* timing) {
  if (misaligned2(scales)) return PA_EINVAL;
  return pa::attend<pa::q8::Format>(q, {k_pages, v_pages, scales, block_table, context_lens, query_start_loc}, true, scale, out, dims,
                                    workspace, workspace_bytes, stream, timing, true);
}

}  // extern "C"
