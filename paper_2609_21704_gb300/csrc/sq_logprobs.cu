// sq_logprobs.cu -- log probabilities of given tokens, entropies and top
// alternatives from rows of fp16 logits.
//
//   x_v = (z_v - max z) / T,  S = sum_v e^x_v
//   log p_v = x_v - log S,  H = log S - sum_v e^x_v x_v / S
#include "sq_serve.h"

namespace sq {

static __device__ unsigned int g_lp_status;

// Total order of (logit, index): largest logit first, lowest index among
// equals (-0 equals 0).  Larger keys come first.
__device__ __forceinline__ uint32_t lp_order16(__half z) {
  uint32_t b = __half_as_ushort(z);
  if (b == 0x8000u) b = 0;
  return b & 0x8000u ? 0xffffu - b : b | 0x8000u;
}
__device__ __forceinline__ unsigned long long lp_key(__half z, uint32_t v) {
  return ((unsigned long long)lp_order16(z) << 32) | (0xffffffffu - v);
}

__device__ __forceinline__ unsigned long long lp_block_max(unsigned long long k, unsigned long long* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long other = __shfl_xor_sync(0xffffffffu, k, o);
    k = other > k ? other : k;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = k;
  __syncthreads();
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) k = red[w] > k ? red[w] : k;
  return k;
}

// One CTA per row; the alternatives one after another.
__global__ void __launch_bounds__(256) logprobs_simple_kernel(const LogprobArgs a) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ unsigned long long red[8];
  __shared__ float fred[2][8];
  const int64_t r = blockIdx.x;
  const __half* z = a.z + r * a.V;
  unsigned long long k = 0;
  bool bad = false;
  for (int64_t v = threadIdx.x; v < a.V; v += blockDim.x) {
    const float f = __half2float(z[v]);
    bad |= isnan(f) || f == INFINITY;
    const unsigned long long key = lp_key(z[v], (uint32_t)v);
    k = key > k ? key : k;
  }
  bad = __syncthreads_or(bad);
  k = lp_block_max(k, red);
  const float m = __half2float(z[0xffffffffu - (uint32_t)k]);
  const bool none = !bad && m == -INFINITY;
  if (bad || none) {
    if (threadIdx.x == 0) {
      atomicOr(&g_lp_status, bad ? SQ_DEV_NONFINITE_LOGIT : SQ_DEV_NO_MASS);
      if (a.logprob) a.logprob[r] = NAN;
      if (a.entropy) a.entropy[r] = NAN;
    }
    for (int i = threadIdx.x; i < a.top; i += blockDim.x) {
      a.top_tokens[r * a.top + i] = -1;
      a.top_logprobs[r * a.top + i] = NAN;
    }
    return;
  }
  // the largest term is 1; the others apart from it, so that a sure row's
  // logarithm keeps them
  const int64_t vmax = 0xffffffffu - (uint32_t)k;
  float S = 0.0f, E = 0.0f;
  for (int64_t v = threadIdx.x; v < a.V; v += blockDim.x) {
    const float x = (__half2float(z[v]) - m) * a.invT;
    if (v == vmax || x == -INFINITY) continue;
    const float e = expf(x);
    S += e;
    E = fmaf(e, -x, E);
  }
  S = warp_sum(S);
  E = warp_sum(E);
  if ((threadIdx.x & 31) == 0) {
    fred[0][threadIdx.x >> 5] = S;
    fred[1][threadIdx.x >> 5] = E;
  }
  __syncthreads();
  S = E = 0.0f;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {
    S += fred[0][w];
    E += fred[1][w];
  }
  const float lse = log1pf(S);
  if (threadIdx.x == 0) {
    if (a.entropy) a.entropy[r] = lse + E / (1.0f + S);
    if (a.tokens) {
      const int64_t t = a.tokens[r];
      const bool ok = t >= 0 && t < a.V;
      if (!ok) atomicOr(&g_lp_status, SQ_DEV_BAD_TOKEN_ID);
      a.logprob[r] = ok ? (__half2float(z[t]) - m) * a.invT - lse : NAN;
    }
  }
  for (int i = 0; i < a.top; ++i) {
    const int64_t v = 0xffffffffu - (uint32_t)k;
    if (threadIdx.x == 0) {
      a.top_tokens[r * a.top + i] = (int32_t)v;
      a.top_logprobs[r * a.top + i] = (__half2float(z[v]) - m) * a.invT - lse;
    }
    unsigned long long n = 0;
    for (int64_t u = threadIdx.x; u < a.V; u += blockDim.x) {
      const unsigned long long key = lp_key(z[u], (uint32_t)u);
      if (key < k && key > n) n = key;
    }
    k = lp_block_max(n, red);
  }
}

cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t st) {
  return launch_pdl(logprobs_simple_kernel, dim3((unsigned)a.R), dim3(256), 0, st, a);
}

cudaError_t take_logprobs_status(uint32_t* bits) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_lp_status, sizeof(v));
  if (e != cudaSuccess) return e;
  if (v) e = cudaMemcpyToSymbol(g_lp_status, &zero, sizeof(zero));
  *bits |= v;
  return e;
}

}  // namespace sq
