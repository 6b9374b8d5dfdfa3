// What the rollout calls share: a head in 4 bits, draft verification, block tables (host-side declarations).
#pragma once

#include "common.cuh"

namespace af {

// ---- head in 4 bits ---------------------------------------------------------------------------
// Eight weights k .. k + 7 of a row share a 32-bit word: weight k + 2 i is digit i of the low half, weight k + 2 i + 1
// digit i of the high half, so that (word >> 4 i) & 0x000f000f is a pair of neighbours.  A digit u stands for
// (u - 8) times the scale of its group.
struct QuantHead {
  const uint32_t* codes;         // [V, d / 8]
  const __nv_bfloat16* scale;    // [V, groups]
  int32_t V, d, group;           // weights per group: 32, 64 or 128; the last group of a row may be short
  int32_t groups() const { return (d + group - 1) / group; }
};
cudaError_t launch_quantize_head(const void* W, int32_t V, int32_t d, int32_t group, void* codes, void* scale, void* values,
                                 cudaStream_t s);
af_status launch_quant_logits(af_ctx* ctx, const void* hidden, const QuantHead& head, int64_t T, void* logits, int32_t type,
                              int64_t pitch, cudaStream_t s);
constexpr int kQuantTokens = 64;  // of one launch (quant_umma.cu)
af_status launch_quant_umma(af_ctx* ctx, const void* hidden, const QuantHead& head, int T, void* logits, int32_t type, int64_t pitch,
                            cudaStream_t s);

// ---- draft verification -----------------------------------------------------------------------
struct LogitRows {
  const void* p;                 // [rows, V], null: none
  int32_t type;                  // AF_F32 or AF_BF16
  int64_t pitch;                 // elements from row to row
};
struct VerifyCall {
  LogitRows target, draft;
  const int32_t* draft_ids;
  const int32_t* cu;
  const float* u_accept;
  const float* u_sample;
  int32_t R, D, V, max_draft;
  float temperature;             // 0: greedy
  int32_t* token;
  float* logp;
  int32_t* n_emitted;
};
af_status reserve_draft_verify(af_ctx* ctx, int32_t R, int32_t max_draft, cudaStream_t s);
af_status launch_draft_verify(af_ctx* ctx, const VerifyCall& c, cudaStream_t s);

// ---- block tables -----------------------------------------------------------------------------
struct SlotsCall {
  const int32_t* length;
  const int32_t* grow;
  const int32_t* held;
  int32_t R;
  int32_t block_size;
  int32_t* table;
  int64_t table_pitch;
  int32_t max_blocks;
  int32_t* free_blocks;
  int32_t n_blocks;
  const int32_t* free_count;
  int32_t* held_out;
  int32_t* free_count_out;
  int32_t* granted;
  int32_t* cu;
  int64_t* slot;
  int32_t* position;
  int64_t capacity;
};
size_t slots_workspace_bytes(int32_t R);
af_status launch_block_slots(af_ctx* ctx, const SlotsCall& c, cudaStream_t s);

}  // namespace af
