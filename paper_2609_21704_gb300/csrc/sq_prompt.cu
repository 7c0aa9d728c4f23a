// sq_prompt.cu -- attention over whole prompts: packed sequences of different
// lengths, causal, grouped heads, each behind the prefix that its cache holds.
//
//   k'_t = fp16(R(pos_t) k_t), cached with v_t at pos_t = pos0 + t
//   out_t = sum_{j <= pos_t} p_tj v_j / sum_j p_tj,
//   p_tj = exp(q'_t . k'_j / sqrt(D)), q'_t = fp16(R(pos_t) q_t)
#include "sq_packed.cuh"

namespace sq {

static __device__ unsigned int g_prompt_status;

// One CTA per row: the rotated queries into the workspace, [Hkv, N, G, D], the
// rotated keys and the values into the caches.  A sequence that does not fit
// its cache writes nothing there, and zeros to its rows of `out`.
__global__ void __launch_bounds__(128) prompt_prepare_kernel(const __half* __restrict__ qkv, const Packed pk,
                                                             int Hq, int Hkv, const RopeFreq rf,
                                                             __half* __restrict__ kc, __half* __restrict__ vc,
                                                             __half* __restrict__ qr, __half* __restrict__ out) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ RopeCS cs[kHeadDim / 2];
  const int64_t row = blockIdx.x;
  const PackedRow pr = packed_row(pk, row);
  if (threadIdx.x == 0 && (pr.bad || (pr.b >= 0 && !pr.ok))) atomicOr(&g_prompt_status, SQ_DEV_BAD_POSITION);
  if (pr.b < 0) return;
  if (!pr.ok) {
    for (int i = threadIdx.x; i < Hq * kHeadDim; i += blockDim.x)
      out[row * Hq * kHeadDim + i] = __ushort_as_half(0);
    return;
  }
  if (threadIdx.x < kHeadDim / 2) cs[threadIdx.x] = rope_cs_pair(pr.pos, rf.f[threadIdx.x]);
  __syncthreads();
  const int G = Hq / Hkv;
  const __half* x = qkv + row * (int64_t)(Hq + 2 * Hkv) * kHeadDim;
  for (int i = threadIdx.x; i < (Hq + 2 * Hkv) * (kHeadDim / 2); i += blockDim.x) {
    const int h = i / (kHeadDim / 2), d = i % (kHeadDim / 2);
    const __half x1 = x[h * kHeadDim + d], x2 = x[h * kHeadDim + d + kHeadDim / 2];
    if (h >= Hq + Hkv) {
      __half* dst = vc + (((int64_t)pr.b * Hkv + h - Hq - Hkv) * pk.max_ctx + pr.pos) * kHeadDim;
      dst[d] = x1;
      dst[d + kHeadDim / 2] = x2;
      continue;
    }
    const float a = __half2float(x1), b = __half2float(x2);
    const RopeCS r = cs[d];
    const __half y1 = __float2half_rn(rope_dot(a, r.c, -b, r.s));
    const __half y2 = __float2half_rn(rope_dot(b, r.c, a, r.s));
    __half* dst = h < Hq ? qr + (((int64_t)(h / G) * pk.N + row) * G + h % G) * kHeadDim
                         : kc + (((int64_t)pr.b * Hkv + h - Hq) * pk.max_ctx + pr.pos) * kHeadDim;
    dst[d] = y1;
    dst[d + kHeadDim / 2] = y2;
  }
}

// One CTA per row, a warp per query head, its keys one after another with the
// running maximum and sum in fp32; a lane holds four dimensions.
__global__ void __launch_bounds__(128) prompt_simple_kernel(const __half* __restrict__ qr, const Packed pk, int Hq,
                                                            int Hkv, const __half* __restrict__ kc,
                                                            const __half* __restrict__ vc,
                                                            __half* __restrict__ out) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = blockIdx.x;
  const PackedRow pr = packed_row(pk, row);
  if (pr.b < 0 || !pr.ok) return;
  const int G = Hq / Hkv, lane = threadIdx.x & 31;
  for (int h = threadIdx.x >> 5; h < Hq; h += blockDim.x >> 5) {
    const int64_t base = ((int64_t)pr.b * Hkv + h / G) * pk.max_ctx * kHeadDim + 4 * lane;
    const __half2* q = reinterpret_cast<const __half2*>(
        qr + (((int64_t)(h / G) * pk.N + row) * G + h % G) * kHeadDim + 4 * lane);
    const float2 q0 = __half22float2(q[0]), q1 = __half22float2(q[1]);
    float m = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = 0; j <= pr.pos; ++j) {
      const __half2* k = reinterpret_cast<const __half2*>(kc + base + (int64_t)j * kHeadDim);
      const __half2* v = reinterpret_cast<const __half2*>(vc + base + (int64_t)j * kHeadDim);
      const float2 k0 = __half22float2(k[0]), k1 = __half22float2(k[1]);
      const float2 v0 = __half22float2(v[0]), v1 = __half22float2(v[1]);
      const float s = warp_sum(q0.x * k0.x + q0.y * k0.y + q1.x * k1.x + q1.y * k1.y) * 0.08838834764831845f;
      if (s == -INFINITY) continue;
      const float mn = fmaxf(m, s);
      const float c = m == -INFINITY ? 0.0f : expf(m - mn), p = expf(s - mn);
      m = mn;
      l = l * c + p;
      o[0] = o[0] * c + p * v0.x;
      o[1] = o[1] * c + p * v0.y;
      o[2] = o[2] * c + p * v1.x;
      o[3] = o[3] * c + p * v1.y;
    }
    __half* dst = out + row * (int64_t)Hq * kHeadDim + (int64_t)h * kHeadDim + 4 * lane;
    for (int e = 0; e < 4; ++e) dst[e] = __float2half_rn(l == 0.0f ? 0.0f : o[e] / l);
  }
}

size_t prompt_workspace_bytes(int B, int64_t N, int Hq, int Hkv, int64_t max_ctx) {
  return (size_t)N * Hq * kHeadDim * sizeof(__half);
}

cudaError_t launch_prompt(const __half* qkv, const Packed& pk, int Hq, int Hkv, double theta, __half* kc,
                          __half* vc, __half* out, void* ws, cudaStream_t st) {
  __half* qr = reinterpret_cast<__half*>(ws);
  cudaError_t e = launch_pdl(prompt_prepare_kernel, dim3((unsigned)pk.N), dim3(128), 0, st, qkv, pk, Hq, Hkv,
                             rope_freq(theta), kc, vc, qr, out);
  if (e != cudaSuccess) return e;
  return launch_pdl(prompt_simple_kernel, dim3((unsigned)pk.N), dim3(128), 0, st, qr, pk, Hq, Hkv, kc, vc, out);
}

cudaError_t take_prompt_status(uint32_t* bits) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_prompt_status, sizeof(v));
  if (e != cudaSuccess) return e;
  if (v) e = cudaMemcpyToSymbol(g_prompt_status, &zero, sizeof(zero));
  *bits |= v;
  return e;
}

}  // namespace sq
