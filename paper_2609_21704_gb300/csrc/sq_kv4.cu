// sq_kv4.cu -- the key/value cache in four bits: append, read back, decode
// attention.
//
// A row (one position of one key/value head) of 128 fp16 values x, the key
// rotated and rounded to fp16 first, is kept as
//   lo = min x, s = fp16((max x - lo) / 15), c = clamp(rint((x - lo) / s), 0, 15),
// every step an IEEE fp32 operation, and stands for c s + lo: 64 bytes of
// codes and two fp16 parameters, 68 bytes against 256.  One scale and one
// lowest value for the whole row keep both out of the products:
//   q . k_j = s_j (q . c_j) + lo_j sum(q)
//   sum_j p_j v_j = sum_j (p_j s_j) c_j + sum_j p_j lo_j.
// Codes: a key's byte i holds dimension 2i in its low half, 2i + 1 in its high
// one.  Values lie in pairs of positions, 128 bytes a pair: two bytes (four
// dimensions) of the even position, then those of the odd one.
#include "sq_packed.cuh"

namespace sq {

static __device__ unsigned int g_kv4_status;

// Codes of one row whose lane holds the fp16 values x[4]; par: scale and lowest.
__device__ __forceinline__ uint32_t kv4_encode(const float x[4], uint32_t& par, bool& fine) {
  float lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
  float hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
  bool ok = true;
#pragma unroll
  for (int e = 0; e < 4; ++e) ok = ok && isfinite(x[e]);
  fine = __all_sync(0xffffffffu, ok);
  if (!fine) {
    par = 0x7fff7fffu;  // NaN: everything read from this row is
    return 0;
  }
  lo = -warp_max(-lo);
  hi = warp_max(hi);
  lo = lo == 0.0f ? 0.0f : lo;
  __half s16 = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.0f));
  if (__half_as_ushort(s16) == 0 && hi > lo) s16 = __ushort_as_half(1);
  const float s = __half2float(s16);
  par = (uint32_t)__half_as_ushort(s16) | ((uint32_t)__half_as_ushort(__float2half_rn(lo)) << 16);
  if (s == 0.0f) return 0;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float c = rintf(__fdiv_rn(__fsub_rn(x[e], lo), s));
    w |= (uint32_t)fminf(fmaxf(c, 0.0f), 15.0f) << (4 * e);
  }
  return w;
}

// One CTA per row, a warp per (key/value head, key or value).
__global__ void __launch_bounds__(128) kv4_append_kernel(const __half* __restrict__ qkv, const Packed pk, int Hq,
                                                         int Hkv, const RopeFreq rf, const KV4Cache c) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ RopeCS cs[kHeadDim / 2];
  const int64_t row = blockIdx.x;
  const PackedRow pr = packed_row(pk, row);
  if (threadIdx.x == 0 && (pr.bad || (pr.b >= 0 && !pr.ok))) atomicOr(&g_kv4_status, SQ_DEV_BAD_POSITION);
  if (pr.b < 0 || !pr.ok) return;
  if (threadIdx.x < kHeadDim / 2) cs[threadIdx.x] = rope_cs_pair(pr.pos, rf.f[threadIdx.x]);
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const __half* xr = qkv + row * (int64_t)(Hq + 2 * Hkv) * kHeadDim;
  for (int i = threadIdx.x >> 5; i < 2 * Hkv; i += blockDim.x >> 5) {
    const bool val = i >= Hkv;
    const int h = val ? i - Hkv : i;
    const int64_t slot = ((int64_t)pr.b * Hkv + h) * pk.max_ctx + pr.pos;
    const __half* src = xr + (int64_t)(Hq + i) * kHeadDim;
    float x[4];
    bool fine;
    uint32_t par, w;
    if (val) {  // dimensions 4 lane ..
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __half2float(src[4 * lane + e]);
      w = kv4_encode(x, par, fine);
      uint16_t* dst = reinterpret_cast<uint16_t*>(c.vc + (slot >> 1) * kHeadDim);
      dst[2 * lane + (slot & 1)] = (uint16_t)w;
    } else {  // dimensions 2 lane, 2 lane + 1 and 64 more
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const RopeCS r = cs[2 * lane + e];
        const float a = __half2float(src[2 * lane + e]), b = __half2float(src[2 * lane + e + kHeadDim / 2]);
        x[e] = __half2float(__float2half_rn(rope_dot(a, r.c, -b, r.s)));
        x[e + 2] = __half2float(__float2half_rn(rope_dot(b, r.c, a, r.s)));
      }
      w = kv4_encode(x, par, fine);
      c.kc[slot * (kHeadDim / 2) + lane] = (uint8_t)w;
      c.kc[slot * (kHeadDim / 2) + lane + 32] = (uint8_t)(w >> 8);
    }
    if (lane == 0) {
      reinterpret_cast<uint32_t*>(val ? c.vp : c.kp)[slot] = par;
      if (!fine) atomicOr(&g_kv4_status, SQ_DEV_NONFINITE_KV);
    }
  }
}

cudaError_t launch_kv4_append(const __half* qkv, const Packed& pk, int Hq, int Hkv, double theta,
                              const KV4Cache& c, cudaStream_t st) {
  return launch_pdl(kv4_append_kernel, dim3((unsigned)pk.N), dim3(128), 0, st, qkv, pk, Hq, Hkv,
                    rope_freq(theta), c);
}

__device__ __forceinline__ float2 kv4_params(const __half* p, int64_t slot) {
  return __half22float2(reinterpret_cast<const __half2*>(p)[slot]);
}

// One CTA per 64 positions of a (sequence, head), a warp per row.
constexpr int kUnpackRows = 64;
__global__ void __launch_bounds__(128) kv4_unpack_kernel(const KV4Cache c, int Hkv, int64_t max_ctx,
                                                         const int32_t* __restrict__ first,
                                                         const int32_t* __restrict__ last, __half* __restrict__ k,
                                                         __half* __restrict__ v) {
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t lo = first[b], hi = last[b];
  if (lo >= hi) return;
  if (lo < 0 || hi > max_ctx) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(&g_kv4_status, SQ_DEV_BAD_POSITION);
    return;
  }
  const int64_t j0 = (int64_t)blockIdx.x * kUnpackRows;
  for (int i = threadIdx.x >> 5; i < kUnpackRows; i += blockDim.x >> 5) {
    const int64_t j = j0 + i;
    if (j < lo || j >= hi) continue;
    const int64_t slot = ((int64_t)b * Hkv + h) * max_ctx + j;
    const float2 kp = kv4_params(c.kp, slot), vp = kv4_params(c.vp, slot);
    const uint32_t kw = reinterpret_cast<const uint16_t*>(c.kc + slot * (kHeadDim / 2))[lane];
    const uint32_t vw = reinterpret_cast<const uint16_t*>(c.vc + (slot >> 1) * kHeadDim)[2 * lane + (slot & 1)];
    __half* kd = k + slot * kHeadDim + 4 * lane;
    __half* vd = v + slot * kHeadDim + 4 * lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      kd[e] = __float2half_rn(fmaf((float)((kw >> (4 * e)) & 15), kp.x, kp.y));
      vd[e] = __float2half_rn(fmaf((float)((vw >> (4 * e)) & 15), vp.x, vp.y));
    }
  }
}

cudaError_t launch_kv4_unpack(const KV4Cache& c, int B, int Hkv, int64_t max_ctx, const int32_t* first,
                              const int32_t* last, __half* k, __half* v, cudaStream_t st) {
  const dim3 grid((unsigned)((max_ctx + kUnpackRows - 1) / kUnpackRows), (unsigned)Hkv, (unsigned)B);
  return launch_pdl(kv4_unpack_kernel, grid, dim3(128), 0, st, c, Hkv, max_ctx, first, last, k, v);
}

// One CTA per new token, a warp per query head; a lane holds dimensions 4 lane ..
__global__ void __launch_bounds__(128) attention_kv4_simple_kernel(const __half* __restrict__ qkv, int T, int Hq,
                                                                   int Hkv, const int32_t* __restrict__ pos0,
                                                                   const RopeFreq rf, const KV4Cache c,
                                                                   int64_t max_ctx, __half* __restrict__ out) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ RopeCS cs[kHeadDim / 2];
  const int64_t row = blockIdx.x;
  const int b = (int)(row / T), t = (int)(row - (int64_t)b * T), lane = threadIdx.x & 31;
  const int64_t p0 = pos0[b];
  const bool ok = p0 >= 0 && p0 + T <= max_ctx;
  if (!ok && threadIdx.x == 0) atomicOr(&g_kv4_status, SQ_DEV_BAD_POSITION);
  const int pos = ok ? (int)p0 + t : -1;
  if (threadIdx.x < kHeadDim / 2) cs[threadIdx.x] = rope_cs_pair(pos, rf.f[threadIdx.x]);
  __syncthreads();
  const int G = Hq / Hkv;
  for (int h = threadIdx.x >> 5; h < Hq; h += blockDim.x >> 5) {
    const __half* x = qkv + row * (int64_t)(Hq + 2 * Hkv) * kHeadDim + (int64_t)h * kHeadDim;
    float q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 4 * lane + e, d1 = d % (kHeadDim / 2);
      const float x1 = __half2float(x[d1]), x2 = __half2float(x[d1 + kHeadDim / 2]);
      const RopeCS r = cs[d1];
      q[e] = d < kHeadDim / 2 ? x1 * r.c.h - x2 * r.s.h : x2 * r.c.h + x1 * r.s.h;
    }
    float m = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = 0; j <= pos; ++j) {
      const int64_t slot = ((int64_t)b * Hkv + h / G) * max_ctx + j;
      const float2 kp = kv4_params(c.kp, slot), vp = kv4_params(c.vp, slot);
      const uint32_t kw = reinterpret_cast<const uint16_t*>(c.kc + slot * (kHeadDim / 2))[lane];
      const uint32_t vw = reinterpret_cast<const uint16_t*>(c.vc + (slot >> 1) * kHeadDim)[2 * lane + (slot & 1)];
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) s = fmaf(q[e], fmaf((float)((kw >> (4 * e)) & 15), kp.x, kp.y), s);
      s = warp_sum(s) * 0.08838834764831845f;
      const float mn = fmaxf(m, s);
      const float f = m == -INFINITY ? 0.0f : expf(m - mn), p = expf(s - mn);
      m = mn;
      l = l * f + p;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = o[e] * f + p * fmaf((float)((vw >> (4 * e)) & 15), vp.x, vp.y);
    }
    __half* dst = out + row * (int64_t)Hq * kHeadDim + (int64_t)h * kHeadDim + 4 * lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = __float2half_rn(l == 0.0f ? 0.0f : o[e] / l);
  }
}

size_t attention_kv4_workspace_bytes(int B, int T, int Hq, int Hkv, int64_t max_ctx) { return 16; }

cudaError_t launch_attention_kv4(const __half* qkv, int B, int T, int Hq, int Hkv, const int32_t* pos0,
                                 double theta, const KV4Cache& c, int64_t max_ctx, __half* out, void* ws,
                                 cudaStream_t st) {
  return launch_pdl(attention_kv4_simple_kernel, dim3((unsigned)(B * T)), dim3(128), 0, st, qkv, T, Hq, Hkv, pos0,
                    rope_freq(theta), c, max_ctx, out);
}

cudaError_t take_kv4_status(uint32_t* bits) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_kv4_status, sizeof(v));
  if (e != cudaSuccess) return e;
  if (v) e = cudaMemcpyToSymbol(g_kv4_status, &zero, sizeof(zero));
  *bits |= v;
  return e;
}

}  // namespace sq
