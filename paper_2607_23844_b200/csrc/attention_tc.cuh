#pragma once
#include "attention.cuh"

namespace oc {
// bf16 queries over a cache in bf16, 8 or 4 bits (attention_tc.cu); the tiles and the split are chosen there.
oc_status launch_attention_tc(oc_ctx*, const AttnParams&, int kv_dtype, int64_t page_rows, cudaStream_t);
// Few rows (attention_few.cu): whether a call has no more of them, and the call.
bool attention_few_rows(const AttnParams&);
oc_status launch_attention_few(oc_ctx*, AttnParams&, int kv_dtype, cudaStream_t);
// The same for fp32 queries (attention_few_f32.cu).
bool attention_few_rows_f32(const AttnParams&);
oc_status launch_attention_few_f32(oc_ctx*, AttnParams&, int kv_dtype, cudaStream_t);
}  // namespace oc
