// Internal launch interface between the C-ABI layer and the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

#include "aflex.h"
#include "aflex_draft.h"
#include "aflex_longctx.h"

namespace aflex {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Library-owned device scratch of the entry points that allocate nothing
// (scratch.hip): kStaticScratchBytes per device, shared by every such call on
// that device. static_scratch returns its device address on the current
// device (looked up once per device, then cached).
constexpr size_t kStaticScratchBytes = size_t(64) << 20;
hipError_t static_scratch(void** ptr);

// Decode attention (attn_decode.hip). attn_shape_fits: the flattened block
// range B * Hkv * ceil(max_context_len / 16) stays below 2^30.
bool attn_shape_fits(const aflex_attn_args& a);
// top > 0: at most that many chosen blocks per (sequence, kv head)
size_t attn_workspace_bytes(const aflex_attn_args& a, int top = 0);
// K/V tiles stream with non-temporal loads: every cached byte is read once,
// alone and next to the FFN's weight stream in the two-stream step alike
// (that step: 2.785 -> 2.730 ms against ordinary loads). The form of the even
// split: kAlone, three 4-wave work-groups per CU with ranges weighted by
// dispatch round (the call has the GPU to itself); kWide, one 12-wave
// work-group per CU (beside the FFN's weight stream, the pipeline step);
// kShared, three 4-wave work-groups per CU with equal ranges (beside other
// work that takes CUs first, the layer step). The workspace is the same.
enum class AttnForm { kAlone, kWide, kShared };
hipError_t launch_attn_decode(const aflex_attn_args& a, void* ws, hipStream_t stream,
                              AttnForm form = AttnForm::kAlone);

// Attention over chosen blocks (attn_decode.hip; workspace: attn_workspace_bytes
// of its attn and top_blocks) and the choice (block_select.hip).
hipError_t launch_attn_sparse(const aflex_attn_sparse_args& s, void* ws, hipStream_t stream);
size_t block_select_workspace_bytes(const aflex_block_select_args& a);
hipError_t launch_block_select(const aflex_block_select_args& a, void* ws, hipStream_t stream);

// Rotation, cache write and block summaries (rope.hip).
hipError_t launch_rope_append(const aflex_rope_args& a, hipStream_t stream);
hipError_t launch_rope_write(const aflex_rope_args& a, hipStream_t stream);
hipError_t launch_block_summary(const aflex_block_summary_args& a, hipStream_t stream);

// Writes into the 8-bit cache (rope_f8.hip), and accepted drafts (cache_accept.hip).
hipError_t launch_rope_append_f8(const aflex_rope_f8_args& a, hipStream_t stream);
hipError_t launch_rope_write_f8(const aflex_rope_f8_args& a, hipStream_t stream);
hipError_t launch_cache_accept(const aflex_cache_accept_args& a, hipStream_t stream);

// Attention of up to max_n query tokens per sequence (attn_rows.hip).
struct RowsShape {
  int B, T, Hq, Hkv, D;
  int max_n;  // bound on a sequence's tokens
  int max_blocks, num_blocks, max_ctx;
  float scale;  // 0: 1 / sqrt(D)
  bool f8;
};
struct RowsTensors {
  const uint16_t* q;
  const void* k_cache;
  const void* v_cache;
  const int8_t* kv_exp;
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* cu_seqlens;  // NULL: a token per sequence
  const uint64_t* masks;      // NULL: chains
  uint16_t* out;
};
bool rows_shape_fits(const RowsShape& s);
size_t rows_workspace_bytes(const RowsShape& s);
hipError_t launch_attn_rows(const RowsShape& s, const RowsTensors& t, void* ws, hipStream_t stream);

// Dense SwiGLU FFN (ffn.hip).
size_t swiglu_workspace_bytes(const aflex_ffn_args& f);
hipError_t launch_swiglu(const aflex_ffn_args& f, void* ws, hipStream_t stream);

// KV-cache append (kv_append.hip) and linear layer (ffn.hip).
hipError_t launch_kv_append(const aflex_kv_append_args& a, hipStream_t stream);
hipError_t launch_kv_write(const aflex_kv_write_args& a, hipStream_t stream);
size_t linear_workspace_bytes(const aflex_linear_args& l);
hipError_t launch_linear(const aflex_linear_args& l, void* ws, hipStream_t stream,
                         const uint16_t* residual = nullptr);

// Top-k MoE FFN (moe.hip).
size_t moe_workspace_bytes(const aflex_ffn_args& f);
// residual (optional, [T, H]) is added to the output in the combine step.
hipError_t launch_moe(const aflex_ffn_args& f, void* ws, hipStream_t stream, const uint16_t* residual = nullptr);
// The two halves of launch_moe: routing (depends only on the logits) and the
// expert computation, with separate workspace blocks.
size_t moe_route_bytes(const aflex_ffn_args& f);
size_t moe_expert_bytes(const aflex_ffn_args& f);
hipError_t launch_moe_route(const aflex_ffn_args& f, void* route_ws, hipStream_t stream);
hipError_t launch_moe_experts(const aflex_ffn_args& f, void* route_ws, void* expert_ws, hipStream_t stream,
                              const uint16_t* residual = nullptr);

// Causal prefill attention (attn_prefill.hip).
hipError_t launch_attn_prefill(const aflex_prefill_args& a, hipStream_t stream);

// RMSNorm + router + MoE block (moe_block.hip).
constexpr int kMaxRouterE = 64;
size_t moe_block_workspace_bytes(const aflex_moe_block_args& m);
hipError_t launch_moe_block(const aflex_moe_block_args& m, void* ws, hipStream_t stream);

}  // namespace aflex
