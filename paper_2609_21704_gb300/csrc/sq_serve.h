// sq_serve.h -- declarations of prompt attention (sq_prompt.cu), the 4-bit
// key/value cache (sq_kv4.cu) and token log probabilities (sq_logprobs.cu).
#pragma once

#include "sq_decoder.h"

namespace sq {

// A row of a packed batch: rows offsets[b] .. offsets[b + 1] - 1 belong to
// sequence b, whose first row is at position pos0[b]; without offsets, T rows
// each.
struct Packed {
  const int32_t* offsets;  // [B + 1] or null
  const int32_t* pos0;     // [B]
  int B;
  int T;                   // rows a sequence (offsets == null)
  int64_t N;               // rows
  int64_t max_ctx;
};

struct KV4Cache {
  uint8_t* kc;  // [B, Hkv, max_ctx, 64]
  __half* kp;   // [B, Hkv, max_ctx, 2]: scale, lowest value
  uint8_t* vc;  // [B, Hkv, max_ctx / 2, 128]
  __half* vp;
};

// sq_prompt.cu
constexpr int64_t kPromptMaxCtx = (int64_t)1 << 17;
size_t prompt_workspace_bytes(int B, int64_t N, int Hq, int Hkv, int64_t max_ctx);
cudaError_t launch_prompt(const __half* qkv, const Packed& pk, int Hq, int Hkv, double theta, __half* kc,
                          __half* vc, __half* out, void* ws, cudaStream_t st);
cudaError_t take_prompt_status(uint32_t* bits);

// sq_kv4.cu
cudaError_t launch_kv4_append(const __half* qkv, const Packed& pk, int Hq, int Hkv, double theta,
                              const KV4Cache& c, cudaStream_t st);
cudaError_t launch_kv4_unpack(const KV4Cache& c, int B, int Hkv, int64_t max_ctx, const int32_t* first,
                              const int32_t* last, __half* k, __half* v, cudaStream_t st);
size_t attention_kv4_workspace_bytes(int B, int T, int Hq, int Hkv, int64_t max_ctx);
cudaError_t launch_attention_kv4(const __half* qkv, int B, int T, int Hq, int Hkv, const int32_t* pos0,
                                 double theta, const KV4Cache& c, int64_t max_ctx, __half* out, void* ws,
                                 cudaStream_t st);
cudaError_t take_kv4_status(uint32_t* bits);

// sq_logprobs.cu
constexpr int kLogprobsMaxTop = 32;
struct LogprobArgs {
  const __half* z;
  const int32_t* tokens;  // or null
  float* logprob;         // [R] or null
  float* entropy;         // [R] or null
  int32_t* top_tokens;    // [R, top]
  float* top_logprobs;    // [R, top]
  int64_t R, V;
  int top;
  float invT;
};
cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t st);
cudaError_t take_logprobs_status(uint32_t* bits);

}  // namespace sq
