// sq_kv4.cu -- the key/value cache in four bits: append, read back, decode
// attention (by mma.sync, and by tcgen05 for many queries over long caches).
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
#include "sq_tcgen.cuh"

#include <algorithm>
#include <mutex>
#include <stddef.h>
#include <type_traits>

namespace sq {

static __device__ unsigned int g_kv4_status;

// Codes (nibble e: x[e]) of one row whose 16 lanes hold eight fp16 values each,
// in pairs; par: scale and lowest.  Smallest and largest run through one shuffle
// (the former negated; a NaN stays one).  A quotient comes from the reciprocal
// (within 2^-19 of the quotient: it is at most 15); only where that leaves the
// rounding open is it divided.
__device__ __forceinline__ uint32_t kv4_encode(const __half2 h[4], uint32_t& par, bool& fine) {
  const __half2 big = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  const __half2 small = __hmin2_nan(__hmin2_nan(h[0], h[1]), __hmin2_nan(h[2], h[3]));
  __half2 ends = __halves2half2(__hneg(__hmin_nan(__low2half(small), __high2half(small))),
                                __hmax_nan(__low2half(big), __high2half(big)));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) ends = __hmax2_nan(ends, __shfl_xor_sync(0xffffffffu, ends, o));
  const float2 e2 = __half22float2(ends);
  const float lo = e2.x == 0.0f ? 0.0f : -e2.x, hi = e2.y;
  fine = fabsf(lo) < INFINITY && fabsf(hi) < INFINITY;
  __half s16 = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.0f));
  if (__half_as_ushort(s16) == 0 && hi > lo) s16 = __ushort_as_half(1);
  const float s = __half2float(s16);
  par = (uint32_t)__half_as_ushort(s16) | ((uint32_t)__half_as_ushort(__float2half_rn(lo)) << 16);
  if (!fine) par = 0x7fff7fffu;  // NaN: everything read from this row is
  if (!fine || s == 0.0f) return 0;
  const float inv = __frcp_rn(s);
  const float one = 12582912.0f;  // 1.5 2^23: its last bits count ones
  uint32_t w = 0;
  float x[8], open = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(h[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = fminf(__fmul_rn(__fsub_rn(x[e], lo), inv), 15.0f);
    const float r = __fadd_rn(q, one);
    open = fmaxf(open, fabsf(q - (r - one)));
    w |= (__float_as_uint(r) & 15u) << (4 * e);
  }
  if (open > 0.4999f) {
    w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      w |= (uint32_t)fminf(rintf(__fdiv_rn(__fsub_rn(x[e], lo), s)), 15.0f) << (4 * e);
  }
  return w;
}

// One CTA a row (several, sharing their tables' computation, waited longer for
// one another: 5493 rows of 8 heads, append and unpack, 35 us with four, 32 with
// one); 16 lanes a
// (key/value head, key or value).  A lane's eight key dimensions are 4u .. 4u + 3
// and 64 more, its rotation entries four that lie 16 entries apart.  Bound: the
// chain of one row (offsets, table, values, ends, codes) and, for thousands of
// rows, instructions: about 40 a value.
constexpr int kAppendThreads = 256;
__global__ void __launch_bounds__(kAppendThreads) kv4_append_kernel(const __half* __restrict__ qkv, const Packed pk,
                                                                    int Hq, int Hkv, const RopeFreq rf,
                                                                    const KV4Cache c) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ RopeCS cs[kHeadDim / 2];  // dimension d at (d % 4) * 16 + d / 4
  __shared__ int seq, pos;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  if (packed_rows<1>(pk, row, &seq, &pos, &g_kv4_status)) return;
  if (seq < 0 || pos < 0) return;
  if (tid < kHeadDim / 2) cs[(tid & 3) * 16 + (tid >> 2)] = rope_cs_pair(pos, rf.f[tid]);
  __syncthreads();
  const int u = tid & 15, per = 2 * Hkv;
  // (the lanes of a warp stay together: 2 Hkv is an even number)
  for (int i = tid >> 4; i < per; i += blockDim.x / 16) {
    const bool val = i >= Hkv;
    const int64_t slot = ((int64_t)seq * Hkv + (val ? i - Hkv : i)) * pk.max_ctx + pos;
    const uint2* src = reinterpret_cast<const uint2*>(qkv + (row * (Hq + per) + Hq + i) * kHeadDim);
    const uint2 v0 = src[val ? 2 * u : u], v1 = src[val ? 2 * u + 1 : u + 16];
    __half2 h[4];
    h[0] = *reinterpret_cast<const __half2*>(&v0.x);
    h[1] = *reinterpret_cast<const __half2*>(&v0.y);
    h[2] = *reinterpret_cast<const __half2*>(&v1.x);
    h[3] = *reinterpret_cast<const __half2*>(&v1.y);
    if (!val) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const RopeCS t0 = cs[2 * p * 16 + u], t1 = cs[(2 * p + 1) * 16 + u];
        const float2 a = __half22float2(h[p]), b = __half22float2(h[p + 2]);
        h[p] = __halves2half2(rope_f16(a.x, t0.c, -b.x, t0.s), rope_f16(a.y, t1.c, -b.y, t1.s));
        h[p + 2] = __halves2half2(rope_f16(b.x, t0.c, a.x, t0.s), rope_f16(b.y, t1.c, a.y, t1.s));
      }
    }
    uint32_t par;
    bool fine;
    const uint32_t w = kv4_encode(h, par, fine);
    uint16_t* dst = val ? reinterpret_cast<uint16_t*>(c.vc + (slot >> 1) * kHeadDim) + (slot & 1)
                        : reinterpret_cast<uint16_t*>(c.kc + slot * (kHeadDim / 2));
    dst[val ? 4 * u : u] = (uint16_t)w;
    dst[val ? 4 * u + 2 : u + 16] = (uint16_t)(w >> 16);
    if (u == 0) {
      reinterpret_cast<uint32_t*>(val ? c.vp : c.kp)[slot] = par;
      if (!fine) atomicOr(&g_kv4_status, SQ_DEV_NONFINITE_KV);
    }
  }
}

cudaError_t launch_kv4_append(const __half* qkv, const Packed& pk, int Hq, int Hkv, double theta,
                              const KV4Cache& c, cudaStream_t st) {
  // 16 threads for each of a row's 2 Hkv parts, 64 at least for its table
  const int threads = Hkv < 2 ? 64 : Hkv < 8 ? 32 * Hkv : kAppendThreads;
  return launch_pdl(kv4_append_kernel, dim3((unsigned)pk.N), dim3((unsigned)threads), 0, st, qkv, pk, Hq, Hkv,
                    rope_freq(theta), c);
}

__device__ __forceinline__ float2 kv4_params(const __half* p, int64_t slot) {
  return __half22float2(reinterpret_cast<const __half2*>(p)[slot]);
}

// One CTA per 32 positions of a (sequence, head); a thread two neighbouring
// positions' eight dimensions of keys and values, 16-byte stores side by side.  5493
// rows of 8 heads: 9.4 us, 4.2 by their bytes; what is written stays in L2 (DRAM 8 %
// busy), and it is bound by instructions (issue 55 %) and the chain of a thread's loads.
// The grid is the caches' capacity (CTAs outside a range end at once).
constexpr int kUnpackRows = 32;
__device__ __forceinline__ uint32_t kv4_half2(uint32_t nibbles, float2 p) {
  // 2^23 + n, less 2^23
  const float a = __uint_as_float(0x4b000000u | (nibbles & 15u)) - 8388608.0f;
  const float b = __uint_as_float(0x4b000000u | ((nibbles >> 4) & 15u)) - 8388608.0f;
  const __half2 r = __floats2half2_rn(fmaf(a, p.x, p.y), fmaf(b, p.x, p.y));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Eight dimensions from four bytes.
__device__ __forceinline__ uint4 kv4_half8(uint32_t w, float2 p) {
  return make_uint4(kv4_half2(w, p), kv4_half2(w >> 8, p), kv4_half2(w >> 16, p), kv4_half2(w >> 24, p));
}
__global__ void __launch_bounds__(256) kv4_unpack_kernel(const KV4Cache c, int Hkv, int64_t max_ctx,
                                                         const int32_t* __restrict__ first,
                                                         const int32_t* __restrict__ last, __half* __restrict__ k,
                                                         __half* __restrict__ v) {
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.z, h = blockIdx.y;
  const int64_t lo = first[b], hi = last[b];
  if (lo >= hi) return;
  if (lo < 0 || hi > max_ctx) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(&g_kv4_status, SQ_DEV_BAD_POSITION);
    return;
  }
  const int64_t j = (int64_t)blockIdx.x * kUnpackRows + (threadIdx.x >> 4) * 2;
  const int u = threadIdx.x & 15;  // dimensions 8 u ..
  if (j + 1 < lo || j >= hi) return;
  const int64_t slot = ((int64_t)b * Hkv + h) * max_ctx + j;
  // (max_ctx is even: both positions of a pair lie in the cache)
  const uint2 vw = reinterpret_cast<const uint2*>(c.vc + (slot >> 1) * kHeadDim)[u];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (j + e < lo || j + e >= hi) continue;
    const uint32_t kw = reinterpret_cast<const uint32_t*>(c.kc + (slot + e) * (kHeadDim / 2))[u];
    // the position's two bytes of every four
    const uint32_t w = __byte_perm(vw.x, vw.y, e ? 0x7632u : 0x5410u);
    reinterpret_cast<uint4*>(k + (slot + e) * kHeadDim)[u] = kv4_half8(kw, kv4_params(c.kp, slot + e));
    reinterpret_cast<uint4*>(v + (slot + e) * kHeadDim)[u] = kv4_half8(w, kv4_params(c.vp, slot + e));
  }
}

cudaError_t launch_kv4_unpack(const KV4Cache& c, int B, int Hkv, int64_t max_ctx, const int32_t* first,
                              const int32_t* last, __half* k, __half* v, cudaStream_t st) {
  const dim3 grid((unsigned)((max_ctx + kUnpackRows - 1) / kUnpackRows), (unsigned)Hkv, (unsigned)B);
  return launch_pdl(kv4_unpack_kernel, grid, dim3(256), 0, st, c, Hkv, max_ctx, first, last, k, v);
}

// ---- attention over the cache ----------------------------------------------------

struct KV4AttnArgs {
  const __half* qkv;
  KV4Cache c;
  const int32_t* pos0;
  __half* out;
  float* part;  // [(B Hkv) nsplit Q kAttnPartStride] where the shares meet in a second launch
  int B, T, Hq, Hkv, G, Q;
  int64_t max_ctx;
  int nsplit;   // CTAs sharing the keys of a (sequence, key/value head, eight queries)
  int cluster;  // they form a cluster and meet in shared memory
  RopeFreq rf;
};

constexpr int kK4Warps = 4, kK4Threads = 32 * kK4Warps;
constexpr int kK4Keys = 32;                   // keys of a warp's step
constexpr int kK4Stages = 3;                  // steps in flight a warp
constexpr int kK4Codes = kK4Keys * 64;        // bytes of a step's key (value) codes
constexpr int kK4Stage = 2 * kK4Codes + 2 * kK4Keys * 4;
constexpr int kK4Rec = kAttnPartStride;       // floats of a query's partial result
template <int R>
struct K4Cfg {
  static constexpr int kQ = 8 * R;            // queries of a CTA
  static constexpr int kOffQ = 0;             // their operands: [R][8 k-steps][32 lanes] 16 bytes
  static constexpr int kOffFac = R * 4096;    // their factors and sums
  static constexpr int kOffCs = kOffFac + 8 * kQ;  // cos and sin of their positions
  static constexpr int kOffRing = kOffCs + kQ * (kHeadDim / 2) * 8;
  static constexpr int kRing = kK4Warps * kK4Stages * kK4Stage;
  static constexpr int kRecs = (kK4Warps + 1) * kQ * kK4Rec * 4;  // over the ring: one a warp, then the CTA's
  static constexpr int kSmem = kOffRing + (kRing > kRecs ? kRing : kRecs);
};

__device__ __forceinline__ void k4_mma(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void k4_cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ float k4_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// x = hi + lo to 22 bits (fp16 terms; a hi that is not finite carries x alone).
__device__ __forceinline__ void k4_split(float x, __half& hi, __half& lo) {
  hi = __float2half_rn(x);
  const float h = __half2float(hi);
  lo = isfinite(h) ? __float2half_rn(x - h) : __ushort_as_half(0);
}
__device__ __forceinline__ uint32_t k4_pack(__half a, __half b) {
  return (uint32_t)__half_as_ushort(a) | ((uint32_t)__half_as_ushort(b) << 16);
}
__device__ __forceinline__ float4 k4_ld_cluster(const float* local, uint32_t rank) {
  uint32_t r;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(local)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(r)
               : "memory");
  return v;
}
__device__ __forceinline__ void k4_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One CTA: 8 R queries (q = g T + t) of a (sequence, key/value head) against a
// share of its keys, four warps taking steps of 32 keys in turn.
//
// A step's codes are 4 KB that lie as the products want them: a lane copies
// (cp.async, two steps ahead, no barrier) and reads 16 bytes of a key's row and
// 16 of two positions' values, and every word of them becomes operands of
// mma.m16n8k16 in the lane itself: keys as the columns of Q K^T in an order of
// dimensions that the queries share, values as the columns of P V with positions
// in pairs, so nothing is moved between lanes or through shared memory.  Scale
// and lowest value of a row enter beside the products.  Codes are n - 8 there, so
// that sums stay as small as the values' own: over a long cache these cancel to a
// hundredth of one, and an offset kept in the codes (64 + n takes two
// instructions in nine fewer a word) left 2^-24 of itself with each addition,
// 4 % of the result behind 30000 tokens.  R = 1, up to eight queries: queries and weights are two fp16 terms each
// (rows 0..7 and 8..15 of a tile), nothing held in 32 bits is rounded to 16.
// R = 2: sixteen queries, rows of their own; queries are two terms (two products),
// a weight relative to its row's maximum is rounded to fp16 (as in
// sq_attention_prompt: with a second term half of the products would be its).
// The running maximum may lag by 2^5 before sums are rescaled.  A power of two, of
// the largest value scale that a query sees, brings weights times value scales into
// fp16's range (steps of 2^-24, against 2^8 to 2^9 for that scale at a weight of one).
// Bound: the products, 96 a step (R = 2; 64 with R = 1) of 16 cycles on each quarter
// of an SM: 456 CTAs over 30000 keys take 196 ns a step of an SM, 150 with R = 1,
// with two CTAs an SM 213 and 162; two or four CTAs' worth of registers and 3 to 9
// shares of the keys change the call by 2 % at most.  R = 1 over a few steps: their
// chain, 4 x 8000 keys, 40 / 8 heads 19.9 us, 1.8 TB/s.
template <int R>
__global__ void __launch_bounds__(kK4Threads, 3) attention_kv4_kernel(const KV4AttnArgs a) {
  using C = K4Cfg<R>;
  griddep_wait();
  griddep_launch_dependents();
  extern __shared__ __align__(128) uint8_t k4_smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const int bh = (int)(blockIdx.x / (unsigned)a.nsplit), split = (int)(blockIdx.x - (unsigned)bh * a.nsplit);
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv, q0 = blockIdx.y * C::kQ, T = a.T;
  const int64_t p0l = a.pos0[b];
  const bool valid = p0l >= 0 && p0l + T <= a.max_ctx;
  if (!valid && split == 0 && blockIdx.y == 0 && tid == 0) atomicOr(&g_kv4_status, SQ_DEV_BAD_POSITION);
  const int p0 = valid ? (int)p0l : 0, len = valid ? p0 + T : 0;
  const int steps = (len + kK4Keys - 1) / kK4Keys;
  const int s0 = (int)((int64_t)split * steps / a.nsplit), s1 = (int)((int64_t)(split + 1) * steps / a.nsplit);

  // this warp's ring; lane pieces of eight keys: 16 bytes of a row each
  const uint32_t ring = smem_u32(k4_smem) + C::kOffRing + warp * (kK4Stages * kK4Stage);
  const uint8_t* slot0 = k4_smem + C::kOffRing + warp * (kK4Stages * kK4Stage);
  const int64_t row = (int64_t)bh * a.max_ctx;
  const uint8_t* kcodes = a.c.kc + row * 64 + lane * 16;
  const uint8_t* vcodes = a.c.vc + row * 64 + t4 * 128 + g * 16;
  const uint8_t* params = reinterpret_cast<const uint8_t*>((lane < 8 ? a.c.kp : a.c.vp) + row * 2) + (lane & 7) * 16;
  auto request = [&](int step, int stage) {
    if (step < s1) {
      const int key = step * kK4Keys;
      const uint32_t dst = ring + stage * kK4Stage + lane * 16;
      // (the cache holds whole groups of 16 keys: the second may lie past its end)
      const int groups = key + 16 < len ? 4 : 2;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < groups) {
          k4_cp16(dst + i * 512, kcodes + (int64_t)key * 64 + i * 512);
          k4_cp16(dst + kK4Codes + i * 512, vcodes + (int64_t)key * 64 + i * 512);
        }
      // parameters: 128 bytes of keys, 128 of values
      if (lane < 16 && (lane & 7) < 2 * groups) k4_cp16(dst + 2 * kK4Codes, params + (int64_t)key * 4);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int step = s0 + warp;
#pragma unroll
  for (int i = 0; i < kK4Stages - 1; ++i) request(step + i * kK4Warps, i);

  // the queries: a warp takes 2 R, rotated in fp32, scaled by a power of two, as
  // operands: k-step kk, half i of lane (g, t4): dimensions 32 t4 + 8 w + e and 4 more,
  // w, e = i'th of (2 kk, 2 kk + 1) by words of eight codes
  __half* qs = reinterpret_cast<__half*>(k4_smem + C::kOffQ);
  float* fac = reinterpret_cast<float*>(k4_smem + C::kOffFac);
  // (a token's table once, by all threads: as many tokens as there are, or queries)
  float2* cs = reinterpret_cast<float2*>(k4_smem + C::kOffCs);
  const int tables = min(T, C::kQ);
  if (s0 < s1)
    for (int i = tid; i < tables * (kHeadDim / 2); i += kK4Threads) {
      const int k = i / (kHeadDim / 2);
      const RopeCS r = rope_cs_pair(p0 + (T <= C::kQ ? k : (q0 + k) % T), a.rf.f[i % (kHeadDim / 2)]);
      cs[i] = make_float2(r.c.h, r.s.h);
    }
  __syncthreads();
  if (s0 < s1)
    for (int i = warp; i < C::kQ; i += kK4Warps) {
      const int q = q0 + i;
      float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // d = lane, lane + 32, lane + 64, lane + 96
      if (q < a.Q) {
        const int hg = q / T, t = q - hg * T;
        const __half* x = a.qkv + (((int64_t)b * T + t) * (a.Hq + 2 * a.Hkv) + kvh * a.G + hg) * kHeadDim + lane;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 r = cs[(T <= C::kQ ? t : i) * (kHeadDim / 2) + lane + 32 * e];
          const float x1 = __half2float(x[32 * e]), x2 = __half2float(x[32 * e + 64]);
          v[e] = x1 * r.x - x2 * r.y;
          v[e + 2] = x2 * r.x + x1 * r.y;
        }
      }
      const float am = warp_max(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))));
      int ex = 10;
      if (am > 0.0f && isfinite(am)) ex = max((int)(__float_as_uint(am) >> 23) - 127, -100);
      const float up = __uint_as_float((uint32_t)(127 + 10 - ex) << 23);  // largest value to [2^10, 2^11)
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __half hi, lo;
        k4_split(v[e] * up, hi, lo);
        sum += __half2float(hi) + __half2float(lo);
        // dimension d = lane + 32 e: t4 = e, w = lane / 8, nibble lane % 8; the pair is nibbles n, n + 4
        const int nib = lane & 7, at = 4 * (lane >> 3) + (nib & 3), kk = at >> 1, half = at & 1;
        // R = 1: tile rows i (high terms) and i + 8 (low); R = 2: row i of the tile of each term
        const int ln = ((R == 1 ? i : i & 7) << 2) + e, up8 = R == 1 ? 0 : i >> 3;
        __half* hi_at = qs + ((kk * 32 + ln) * 4 + 2 * half + up8) * 2 + (nib >> 2);
        __half* lo_at = R == 1 ? qs + ((kk * 32 + ln) * 4 + 2 * half + 1) * 2 + (nib >> 2) : hi_at + 2048;
        *hi_at = hi;
        *lo_at = lo;
      }
      sum = warp_sum(sum);
      if (lane == 0) {
        // scores in units of log 2
        fac[i] = 0.08838834764831845f * 1.4426950408889634f * __uint_as_float((uint32_t)(127 + ex - 10) << 23);
        fac[C::kQ + i] = sum;
      }
    }
  __syncthreads();
  float fq[R], qsum[R];
  int lim[R];  // the last position a row sees
  const uint4* qop = reinterpret_cast<const uint4*>(k4_smem + C::kOffQ) + lane;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    fq[r] = s0 < s1 ? fac[8 * r + g] : 0.0f;
    qsum[r] = s0 < s1 ? fac[C::kQ + 8 * r + g] : 0.0f;
    lim[r] = p0 + (q0 + 8 * r + g) % T;
  }

  float o[16][4], m[R], l[R], zl[R];
  float vcap[R], vup[R];  // scales of the values a query sees: up to vcap; vup brings them to 2^9
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = zl[r] = vcap[r] = 0.0f;
    vup[r] = 1.0f;
  }

  for (int it = 0; step < s1; ++it, step += kK4Warps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kK4Stages - 2) : "memory");
    __syncwarp();  // the parameters are other lanes' copies
    const uint8_t* sl = slot0 + (it % kK4Stages) * kK4Stage;
    const bool edge = (step + 1) * kK4Keys > p0 + 1;
    float sc[R][4][2], mx[R], vm[R];
    {
      // scores: four columns' tiles of eight keys, two chains of products at a time
      float s[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
      for (int np = 0; np < 4; np += 2) {
        const uint4 ka = *reinterpret_cast<const uint4*>(sl + np * 512 + lane * 16);
        const uint4 kb = *reinterpret_cast<const uint4*>(sl + np * 512 + 512 + lane * 16);
        const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t ra[4], rb[4];
          int4x8_to_f16x2(wa[i], ra);
          int4x8_to_f16x2(wb[i], rb);
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int term = 0; term < R; ++term) {
              const uint4 qv = qop[(term * 8 + 2 * i + half) * 32];
              const uint32_t qa[4] = {qv.x, qv.y, qv.z, qv.w};
              k4_mma(s[np], qa, ra[2 * half], ra[2 * half + 1]);
              k4_mma(s[np + 1], qa, rb[2 * half], rb[2 * half + 1]);
            }
        }
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const uint2 kp = *reinterpret_cast<const uint2*>(sl + 2 * kK4Codes + n * 32 + t4 * 8);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 k2 = __half22float2(*reinterpret_cast<const __half2*>(e ? &kp.y : &kp.x));
          const float k0 = fmaf(8.0f, k2.x, k2.y);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float raw = R == 1 ? s[n][e] + s[n][e + 2] : s[n][2 * r + e];
            sc[r][n][e] = fq[r] * fmaf(k2.x, raw, k0 * qsum[r]);
          }
        }
      }
    }
    float ws[4][2], wl[4][2];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint2 vp = *reinterpret_cast<const uint2*>(sl + 2 * kK4Codes + 128 + n * 32 + t4 * 8);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 v2 = __half22float2(*reinterpret_cast<const __half2*>(e ? &vp.y : &vp.x));
        ws[n][e] = v2.x;
        wl[n][e] = fmaf(8.0f, v2.x, v2.y);
      }
    }
    if (edge) {  // rows that a query does not see, and those past the last token (they may hold anything)
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = step * kK4Keys + 8 * n + 2 * t4 + e;
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (key > lim[r]) sc[r][n][e] = -INFINITY;
          if (key >= len || (R == 1 && key > lim[0])) ws[n][e] = wl[n][e] = 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mx[r] = -INFINITY;
      vm[r] = 0.0f;
    }
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        vm[0] = fmaxf(vm[0], ws[n][e]);
#pragma unroll
        for (int r = 0; r < R; ++r) mx[r] = fmaxf(mx[r], sc[r][n][e]);
      }
    if (R > 1) {
      vm[R - 1] = vm[0];
      if (edge) {  // (of the rows that each of the two queries sees)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          vm[r] = 0.0f;
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (step * kK4Keys + 8 * n + 2 * t4 + e <= lim[r]) vm[r] = fmaxf(vm[r], ws[n][e]);
        }
      }
    }
    bool grown = false;
#pragma unroll
    for (int r = 0; r < R; ++r) grown = grown || vm[r] > vcap[r] || mx[r] - m[r] > 5.0f;
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float fv = 1.0f;
        vm[r] = fmaxf(vm[r], __shfl_xor_sync(0xffffffffu, vm[r], 1));
        vm[r] = fmaxf(vm[r], __shfl_xor_sync(0xffffffffu, vm[r], 2));
        if (vm[r] > vcap[r]) {
          // the power of two above vm becomes 2^9: weights up to 2^5 stay below 2^15
          const float cap = __uint_as_float(((__float_as_uint(vm[r]) >> 23) + 1) << 23);
          const float up = 512.0f / cap;
          fv = up / vup[r];
          vcap[r] = cap;
          vup[r] = up;
        }
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
        const float mn = fmaxf(m[r], mx[r]);
        float f = m[r] == -INFINITY ? 0.0f : k4_ex2(m[r] - mn);
        m[r] = mn;
        l[r] *= f;
        zl[r] *= f;
        f *= fv;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          o[i][2 * r] *= f;
          o[i][2 * r + 1] *= f;
          if (R == 1) {
            o[i][2] *= f;
            o[i][3] *= f;
          }
        }
      }
    }
    uint32_t pa[2][4];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float mm = m[r] == -INFINITY ? 0.0f : m[r];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        __half hi[2], lo[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p = k4_ex2(sc[r][n][e] - mm);
          l[r] += p;
          float w = ws[n][e] * vup[r], wlow = wl[n][e];
          // (a row that the one query sees and the other does not may hold a NaN)
          if (R > 1 && edge && sc[r][n][e] == -INFINITY) w = wlow = 0.0f;
          const float x = p * w;
          zl[r] = fmaf(p, wlow, zl[r]);
          if (R == 1) {
            hi[e] = __float2half_rn(x);  // (below 2^15)
            lo[e] = __float2half_rn(x - __half2float(hi[e]));
          } else {
            hi[e] = __float2half_rn(x);
          }
        }
        if (R == 1) {
          pa[n >> 1][2 * (n & 1)] = k4_pack(hi[0], hi[1]);
          pa[n >> 1][2 * (n & 1) + 1] = k4_pack(lo[0], lo[1]);
        } else {
          pa[n >> 1][2 * (n & 1) + r] = k4_pack(hi[0], hi[1]);
        }
      }
    }
#pragma unroll
    for (int np = 0; np < 2; ++np) {
      const uint4 va = *reinterpret_cast<const uint4*>(sl + kK4Codes + np * 1024 + lane * 16);
      const uint4 vb = *reinterpret_cast<const uint4*>(sl + kK4Codes + np * 1024 + 512 + lane * 16);
      const uint32_t wa[4] = {va.x, va.y, va.z, va.w}, wb[4] = {vb.x, vb.y, vb.z, vb.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t ra[4], rb[4];
        int4x8_to_f16x2(wa[u], ra);
        int4x8_to_f16x2(wb[u], rb);
#pragma unroll
        for (int e = 0; e < 4; ++e) k4_mma(o[4 * u + e], pa[np], ra[e], rb[e]);
      }
    }
    __syncwarp();  // every lane has read the parameters
    request(step + (kK4Stages - 1) * kK4Warps, (it + kK4Stages - 1) % kK4Stages);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();

  // ---- records (m, l, -, -, o[D]) over the ring: a warp's, then the CTA's
  float* rec = reinterpret_cast<float*>(k4_smem + C::kOffRing);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float down = 1.0f / vup[r];
#pragma unroll
    for (int i = 1; i < 4; i <<= 1) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], i);
      zl[r] += __shfl_xor_sync(0xffffffffu, zl[r], i);
    }
    float* to = rec + (warp * C::kQ + 8 * r + g) * kK4Rec;
    if (t4 == 0) {
      // (natural units, as attention_combine_kernel has them, which takes sums above
      // zero only: where weights are NaN, and so the values' sums are, the record has to count)
      to[0] = isnan(l[r]) ? 0.0f : m[r] * 0.6931471805599453f;
      to[1] = isnan(l[r]) ? 1.0f : l[r];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float* t = o[4 * u + k];
          x[k] = fmaf(R == 1 ? t[e] + t[e + 2] : t[2 * r + e], down, zl[r]);
        }
        *reinterpret_cast<float4*>(to + 4 + 16 * (2 * t4 + e) + 4 * u) = make_float4(x[0], x[1], x[2], x[3]);
      }
  }
  __syncthreads();
  const int nq = min(C::kQ, a.Q - q0);
  float* mine = rec + kK4Warps * C::kQ * kK4Rec;
  for (int i = tid; i < nq * (kHeadDim / 4); i += kK4Threads) {
    const int q = i / (kHeadDim / 4), d4 = i % (kHeadDim / 4);
    float M = -INFINITY, L = 0.0f;
    float4 O = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kK4Warps; ++w) M = fmaxf(M, rec[(w * C::kQ + q) * kK4Rec]);
#pragma unroll
    for (int w = 0; w < kK4Warps; ++w) {
      const float* r = rec + (w * C::kQ + q) * kK4Rec;
      if (r[0] == -INFINITY) continue;
      const float f = expf(r[0] - M);
      const float4 v = *reinterpret_cast<const float4*>(r + 4 + 4 * d4);
      L = fmaf(f, r[1], L);
      O.x = fmaf(f, v.x, O.x);
      O.y = fmaf(f, v.y, O.y);
      O.z = fmaf(f, v.z, O.z);
      O.w = fmaf(f, v.w, O.w);
    }
    float* r = mine + q * kK4Rec;
    if (d4 == 0) {
      r[0] = M;
      r[1] = L;
    }
    *reinterpret_cast<float4*>(r + 4 + 4 * d4) = O;
  }
  __syncthreads();

  if (!a.cluster && a.nsplit > 1) {  // to the workspace, merged by attention_combine_kernel
    float* part = a.part + (((int64_t)bh * a.nsplit + split) * a.Q + q0) * kK4Rec;
    for (int i = tid; i < nq * (kK4Rec / 4); i += kK4Threads)
      reinterpret_cast<float4*>(part)[i] = reinterpret_cast<const float4*>(mine)[i];
    return;
  }
  // ---- the cluster's records in rank order; rank r writes its share
  const int S = a.nsplit;
  if (S > 1) k4_cluster_sync();
  const int n = nq * (kHeadDim / 4);
  const int i0 = (int)((int64_t)split * n / S), i1 = (int)((int64_t)(split + 1) * n / S);
  for (int i = i0 + tid; i < i1; i += kK4Threads) {
    const int q = i / (kHeadDim / 4), d4 = i % (kHeadDim / 4);
    float M = -INFINITY, L = 0.0f;
    float4 O = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int r0 = 0; r0 < S; r0 += 8) {
      float4 ml[8], ov[8];  // eight ranks' records in flight
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r0 + u < S) {
          ml[u] = k4_ld_cluster(mine + q * kK4Rec, (uint32_t)(r0 + u));
          ov[u] = k4_ld_cluster(mine + q * kK4Rec + 4 + 4 * d4, (uint32_t)(r0 + u));
        }
      float Mn = M;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r0 + u < S) Mn = fmaxf(Mn, ml[u].x);
      if (Mn == -INFINITY) continue;
      const float f0 = M == -INFINITY ? 0.0f : expf(M - Mn);
      L *= f0;
      O.x *= f0; O.y *= f0; O.z *= f0; O.w *= f0;
      M = Mn;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r0 + u < S && ml[u].x != -INFINITY) {
          const float f = expf(ml[u].x - M);
          L = fmaf(f, ml[u].y, L);
          O.x = fmaf(f, ov[u].x, O.x);
          O.y = fmaf(f, ov[u].y, O.y);
          O.z = fmaf(f, ov[u].z, O.z);
          O.w = fmaf(f, ov[u].w, O.w);
        }
    }
    const int qq = q0 + q, hg = qq / T, t = qq - hg * T;
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    __half* dst = a.out + (((int64_t)b * T + t) * a.Hq + kvh * a.G + hg) * kHeadDim + 4 * d4;
    *reinterpret_cast<uint2*>(dst) =
        make_uint2(k4_pack(__float2half_rn(O.x * inv), __float2half_rn(O.y * inv)),
                   k4_pack(__float2half_rn(O.z * inv), __float2half_rn(O.w * inv)));
  }
  if (S > 1) k4_cluster_sync();  // no CTA leaves while another reads its records
}

// ---- many queries over long caches: tcgen05 ----------------------------------------

// One CTA an SM: N queries (32 or 48) of a (sequence, key/value head) against a share
// of its keys, in tiles of 128.  Transposed products, so that keys and dimensions
// fill the 128 rows of the tensor core and queries are its columns:
//   S^T = K Q^T (a key's codes a row, queries in two fp16 terms: two products),
//   O^T += V^T P^T (a dimension's codes a row).
// A warp copies the cache's tiles as they are (three in flight; loads into registers
// would be waited for by the fence before every hand-over).  Two groups of four warps
// turn the keys' and the values' codes into fp16 operands, once for all queries.
// Four warps have a key a thread: its scale and lowest value enter beside the
// products, its weights times its value's scale go to shared memory as fp16, and it
// keeps sums of weights (and of weights times lowest values) for every query to the
// end.  The queries' running maxima lie in shared memory, may lag by 2^5, and change
// where the four warps agree.  One thread issues the products.
// attention_kv4_kernel converts a code for every sixteen queries and is bound by
// mma.sync, 16 cycles an m16n8k16 on each quarter of an SM: 16 x 5 tokens behind
// 30000, 28 / 4 heads, 282 us.  Here 152, 1.2 us a tile.  What that is made of (taken
// with three rounds of CTAs, 163 us in all): without copies, conversion and softmax
// 140, with a third of the products besides 105; the rest are hand-overs (weights
// written, products, their place free).  Two places for the weights and two tiles of
// copies in flight instead of one and three: 182; one group for keys and values 196;
// codes loaded into registers 302.
constexpr int kT4Keys = 128, kT4Threads = 512;
constexpr int kT4Tile = kT4Keys * kHeadDim * 2;  // fp16 operands of a tile's keys (or values)
constexpr int kT4Max = 48;                       // queries of a CTA
// What the tensor core adds to a sum it cuts where an fp32 addition rounds, and the
// codes' part of the values does not cancel as the values do (their lowest ones come
// beside it): 117 tiles in one sum were off by 2.4e-4 of the result, 34 by 0.7e-4.  So
// tiles go to six sums in turn, which are added at the end, and no CTA takes more than
// 24 tiles to each.
constexpr int kT4Sums = 6, kT4MaxTiles = 24 * kT4Sums;
constexpr int kT4OffV = 2 * kT4Tile, kT4OffP = 4 * kT4Tile;
constexpr int kT4P = kT4Keys * 128;              // weights of a tile: 64 queries' places a key
constexpr int kT4OffQ = kT4OffP + kT4P;      // two terms x two halves of the dimensions
constexpr int kT4QRows = kT4Max * 128;           // bytes of a term's half
constexpr int kT4OffC = kT4OffQ + 4 * kT4QRows;  // tiles of the cache as it is: codes, then parameters
constexpr int kT4Stages = 3;
constexpr int kT4Codes = kT4Keys * 64, kT4Stage = 2 * kT4Codes + 2 * kT4Keys * 4;
constexpr int kT4OffS = kT4OffC + kT4Stages * kT4Stage;
struct T4Shared {
  float m[kT4Max], fac[kT4Max];  // running maxima (units of log 2); what sums of weights are rescaled by
  float cap[kT4Max], up[kT4Max], fo[kT4Max];  // scales of the values a query sees: up to cap; up brings
                                              // them to 2^9; what sums of values are rescaled by
  alignas(16) float neg[kT4Max];
  alignas(16) float qsum[kT4Max];
  int lim[kT4Max];               // the last position a query sees
  float wm[4][kT4Max], wv[4][kT4Max];  // maxima of the warps: scores, value scales
  float total[2][kT4Max];
  int amax;                      // largest finite |query value|, as bits
  uint64_t c_full[kT4Stages], c_empty[kT4Stages], k_full[2], v_full[2], s_full[2], p_ready[2], pv_done[2], drain;
  uint32_t tmem;
  int dead;
};
constexpr int kT4Smem = kT4OffS + (int)sizeof(T4Shared) + 1024;
static_assert(kT4Smem <= 227 * 1024, "fits an SM");

__device__ __forceinline__ uint64_t t4_desc_mn(uint32_t saddr) {  // 64 columns a row, an atom of 8 rows 1024 on
  uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ uint32_t t4_any(uint32_t x) {  // of the 128 softmax threads
  uint32_t r;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbar.red.or.pred q, 1, 128, p;\nselp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"(x)
      : "memory");
  return r;
}
// Where 16 bytes go: words' dimensions 8 W .. 8 W + 7 of a row, in the order 0 4 1 5 2 6
// 3 7 of the codes' conversion.  Halves of the dimensions 64 columns each; the second
// has its words in another order, so that eight lanes' stores meet eight bank groups.
__device__ __forceinline__ uint32_t t4_piece(int row, int W) {
  const int half = W >> 3, piece = (W & 4) | ((W & 3) ^ (half * 2));
  return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4));
}

template <int N>
__global__ void __launch_bounds__(kT4Threads, 1) attention_kv4_tc_kernel(const KV4AttnArgs a) {
  extern __shared__ uint8_t t4_raw[];
  uint8_t* smem = t4_raw + (((smem_u32(t4_raw) + 1023u) & ~1023u) - smem_u32(t4_raw));
  T4Shared* s = reinterpret_cast<T4Shared*>(smem + kT4OffS);
  const uint32_t base = smem_u32(smem), bars = base + kT4OffS;
#define T4_BAR(member) (bars + (uint32_t)offsetof(T4Shared, member))
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kT4Stages; ++i) {
      mbar_init(&s->c_full[i], 1);
      mbar_init(&s->c_empty[i], 12);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s->k_full[i], 4);
      mbar_init(&s->v_full[i], 4);
      mbar_init(&s->s_full[i], 1);
      mbar_init(&s->p_ready[i], 4);
      mbar_init(&s->pv_done[i], 1);
    }
    mbar_init(&s->drain, 1);
    s->dead = 0;
    s->amax = 0;
    fence_mbar_init();
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s->tmem)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&s->tmem;  // S^T at 0 and 64, O^T's places from 128 on, 64 columns each
  griddep_wait();
  griddep_launch_dependents();

  const int bh = (int)(blockIdx.x / (unsigned)a.nsplit), split = (int)(blockIdx.x - (unsigned)bh * a.nsplit);
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv, q0 = blockIdx.y * N, T = a.T, nq = min(N, a.Q - q0);
  const int64_t p0l = a.pos0[b];
  const bool valid = p0l >= 0 && p0l + T <= a.max_ctx;
  if (!valid && split == 0 && blockIdx.y == 0 && tid == 0) atomicOr(&g_kv4_status, SQ_DEV_BAD_POSITION);
  const int p0 = valid ? (int)p0l : 0, len = valid ? p0 + T : 0;
  const int tiles = (len + kT4Keys - 1) / kT4Keys;
  const int t0 = (int)((int64_t)split * tiles / a.nsplit), t1 = (int)((int64_t)(split + 1) * tiles / a.nsplit);
  const int n = t1 - t0;
  const int64_t row = (int64_t)bh * a.max_ctx;  // of the cache

  // ---- the queries, rotated in fp32, by one power of two for all (the largest to
  // [2^10, 2^11)), as two fp16 terms; warps 0 .. 7 take every eighth
  float2* cs = reinterpret_cast<float2*>(smem + kT4OffP);  // (the weights come later)
  if (n > 0) {
    for (int i = tid; i < min(T, N) * (kHeadDim / 2); i += kT4Threads) {
      const int k = i / (kHeadDim / 2);
      const RopeCS r = rope_cs_pair(p0 + (T <= N ? k : (q0 + k) % T), a.rf.f[i % (kHeadDim / 2)]);
      cs[i] = make_float2(r.c.h, r.s.h);
    }
    __syncthreads();
    float v[N / 8][4];
    if (warp < 8) {
#pragma unroll
      for (int j = 0; j < N / 8; ++j) {
        const int i = warp + 8 * j, q = q0 + i;
        v[j][0] = v[j][1] = v[j][2] = v[j][3] = 0.0f;  // d = lane + 32 e
        if (i < nq) {
          const int hg = q / T, t = q - hg * T;
          const __half* x = a.qkv + (((int64_t)b * T + t) * (a.Hq + 2 * a.Hkv) + kvh * a.G + hg) * kHeadDim + lane;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 r = cs[(T <= N ? t : i) * (kHeadDim / 2) + lane + 32 * e];
            const float x1 = __half2float(x[32 * e]), x2 = __half2float(x[32 * e + 64]);
            v[j][e] = x1 * r.x - x2 * r.y;
            v[j][e + 2] = x2 * r.x + x1 * r.y;
          }
        }
        float am = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (isfinite(v[j][e])) am = fmaxf(am, fabsf(v[j][e]));
        am = warp_max(am);
        if (lane == 0) atomicMax(&s->amax, __float_as_int(am));
      }
    }
    __syncthreads();
    const int ex = s->amax ? max((s->amax >> 23) - 127, -100) : 10;
    const float up = __uint_as_float((uint32_t)(127 + 10 - ex) << 23);
    if (warp < 8) {
#pragma unroll
      for (int j = 0; j < N / 8; ++j) {
        const int i = warp + 8 * j;
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          __half hi, lo;
          k4_split(v[j][e] * up, hi, lo);
          sum += __half2float(hi) + __half2float(lo);
          const int d = lane + 32 * e, k = d & 7, half = d >> 6;
          const uint32_t at = kT4OffQ + half * kT4QRows + t4_piece(i, d >> 3) + ((k & 3) * 2 + (k >> 2)) * 2;
          *reinterpret_cast<__half*>(smem + at) = hi;
          *reinterpret_cast<__half*>(smem + at + 2 * kT4QRows) = lo;
        }
        sum = warp_sum(sum);
        if (lane == 0) {
          s->qsum[i] = sum;
          s->lim[i] = p0 + (q0 + i) % T;
          s->m[i] = -INFINITY;
          s->neg[i] = INFINITY;
          s->cap[i] = 0.0f;
          s->up[i] = 1.0f;
        }
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // scores in units of log 2
  const float unit = 0.08838834764831845f * 1.4426950408889634f *
                     __uint_as_float((uint32_t)(127 + (s->amax ? max((s->amax >> 23) - 127, -100) : 10) - 10) << 23);
  __syncthreads();

  // registers: 512 threads x 128 at launch; the softmax warps take 208, the others
  // keep 96 (128 x 208 + 384 x 96 <= 512 x 128)
  if (warp >= 4) {
   asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
   if (warp == 13) {
    if (lane == 0) {
      // ------------------------------------------------------------- copies
      int t = 0;
      bool fine = true;
      for (; t < n; ++t) {
        const int p = t % kT4Stages;
        if (t >= kT4Stages &&
            !(fine = tc_wait(T4_BAR(c_empty) + 8 * p, ((t / kT4Stages) & 1) ^ 1, &s->dead, &g_kv4_status)))
          break;
        // (the cache may end inside the tile, after a group of 16)
        const int64_t key = (int64_t)(t0 + t) * kT4Keys;
        const uint32_t rows = (uint32_t)min((int64_t)kT4Keys, a.max_ctx - key);
        uint8_t* to = smem + kT4OffC + p * kT4Stage;
        mbar_arrive_expect_tx(&s->c_full[p], rows * 136);
        bulk_g2s(to, a.c.kc + (row + key) * 64, rows * 64, &s->c_full[p]);
        bulk_g2s(to + kT4Codes, a.c.vc + (row + key) * 64, rows * 64, &s->c_full[p]);
        bulk_g2s(to + 2 * kT4Codes, a.c.kp + (row + key) * 2, rows * 4, &s->c_full[p]);
        bulk_g2s(to + 2 * kT4Codes + kT4Keys * 4, a.c.vp + (row + key) * 2, rows * 4, &s->c_full[p]);
      }
      if (!fine)  // what was asked for has to arrive
        for (int i = max(t - kT4Stages, 0); i < t; ++i)
          mbar_wait_bounded(&s->c_full[i % kT4Stages], (i / kT4Stages) & 1, 1u << 20);
    }
   } else if (warp == 12) {
    if (lane == 0) {
      // ------------------------------------------------------------- products
      const uint32_t id_qk = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((128u >> 4) << 24);
      const uint32_t id_pv = id_qk | (1u << 16);  // of the weights queries run
      bool fine = true;
      for (int t = 0; fine && t <= n; ++t) {
        if (n == 0) break;
        if (t < n) {
          const int p = t & 1;
          if (!(fine = tc_wait(T4_BAR(k_full) + 8 * p, (t >> 1) & 1, &s->dead, &g_kv4_status))) break;
          tc_fence_after();
          const uint64_t kd = sw128_desc(base + p * kT4Tile), qd = sw128_desc(base + kT4OffQ);
#pragma unroll
          for (int term = 0; term < 2; ++term)
#pragma unroll
            for (int kk = 0; kk < kHeadDim / 16; ++kk)
              tc_mma_f16(tmem + 64 * p, kd + (kk >> 2) * (kT4Tile / 2 / 16) + (kk & 3) * 2,
                         qd + term * (2 * kT4QRows / 16) + (kk >> 2) * (kT4QRows / 16) + (kk & 3) * 2, id_qk,
                         term + kk > 0);
          tc_commit_at(T4_BAR(s_full) + 8 * p);
        }
        if (t > 0) {
          const int p = (t - 1) & 1, ph = ((t - 1) >> 1) & 1;
          if (!(fine = tc_wait(T4_BAR(v_full) + 8 * p, ph, &s->dead, &g_kv4_status) &&
                       tc_wait(T4_BAR(p_ready) + 8 * p, ph, &s->dead, &g_kv4_status)))
            break;
          tc_fence_after();
          const uint64_t vd = sw128_desc(base + kT4OffV + p * kT4Tile), pd = t4_desc_mn(base + kT4OffP);
#pragma unroll
          for (int kk = 0; kk < kT4Keys / 16; ++kk)
            tc_mma_f16(tmem + 128 + 64 * ((t - 1) % kT4Sums), vd + (kk >> 2) * (kT4Tile / 2 / 16) + (kk & 3) * 2,
                       pd + kk * (16 * 128 / 16), id_pv, t > kT4Sums || kk > 0);
          tc_commit_at(T4_BAR(pv_done) + 8 * p);
        }
      }
      if (!fine) {  // what was issued still reads shared memory and writes TMEM
        tc_commit_at(T4_BAR(drain));
        mbar_wait_bounded(&s->drain, 0u, 1u << 20);
      }
    }
   } else if (warp < 8) {
    // --------------------------------------------------------------- keys' codes to operands
    const int ct = tid - 128, t4 = ct & 3;
    for (int t = 0; t < n; ++t) {
      const int p = t & 1, ph = (t >> 1) & 1, c_at = t % kT4Stages;
      const uint8_t* from = smem + kT4OffC + c_at * kT4Stage;
      tc_wait(T4_BAR(c_full) + 8 * c_at, (t / kT4Stages) & 1, &s->dead, &g_kv4_status);
      uint4 c[4];  // pieces ct + 128 i: key / 4, 16 bytes of its 64
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = *reinterpret_cast<const uint4*>(from + (ct + 128 * i) * 16);
      __syncwarp();
      if (lane == 0) tc_arrive(T4_BAR(c_empty) + 8 * c_at);
      // (the tile two before is done with)
      if (t >= 2) tc_wait(T4_BAR(s_full) + 8 * p, ph ^ 1, &s->dead, &g_kv4_status);
      uint8_t* to = smem + p * kT4Tile + (t4 >> 1) * (kT4Tile / 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t o[4];
          int4x8_to_f16x2(w[j], o);
          *reinterpret_cast<uint4*>(to + t4_piece((ct + 128 * i) >> 2, 4 * t4 + j)) =
              make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) tc_arrive(T4_BAR(k_full) + 8 * p);
    }
   } else if (warp < 12) {
    // --------------------------------------------------------------- values' codes to operands
    const int u = lane & 7, kg = (warp - 8) * 4 + (lane >> 3);  // dimensions 16 u .. of eight keys
    for (int t = 0; t < n; ++t) {
      const int p = t & 1, ph = (t >> 1) & 1, c_at = t % kT4Stages;
      const uint8_t* from = smem + kT4OffC + c_at * kT4Stage + kT4Codes + kg * 512 + u * 16;
      tc_wait(T4_BAR(c_full) + 8 * c_at, (t / kT4Stages) & 1, &s->dead, &g_kv4_status);
      uint4 c[4];  // four pairs of positions
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = *reinterpret_cast<const uint4*>(from + i * 128);
      __syncwarp();
      if (lane == 0) tc_arrive(T4_BAR(c_empty) + 8 * c_at);
      if (t >= 2) tc_wait(T4_BAR(pv_done) + 8 * p, ph ^ 1, &s->dead, &g_kv4_status);
      // dimension 16 u + 4 j + e in row (4 j + e) 8 + u: eight lanes, eight bank groups
      uint8_t* to = smem + kT4OffV + p * kT4Tile + (kg >> 3) * (kT4Tile / 2) + u * 128 + (((kg & 7) ^ u) << 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t o[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          int4x8_to_f16x2(j == 0 ? c[i].x : j == 1 ? c[i].y : j == 2 ? c[i].z : c[i].w, o[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint4*>(to + (4 * j + e) * 1024) = make_uint4(o[0][e], o[1][e], o[2][e], o[3][e]);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) tc_arrive(T4_BAR(v_full) + 8 * p);
    }
   }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // --------------------------------------------------------------- softmax: a key a thread
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const int first = p0;  // a position that every query sees
    unsigned long long l2[N / 2], z2[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) l2[i] = z2[i] = 0;
    float vcap = 0.0f, vup = 1.0f;  // every query's before the first position that one does not see
    for (int t = 0; t < n; ++t) {
      const int p = t & 1, key = (t0 + t) * kT4Keys + tid;  // (below 2^17)
      const bool edge = (t0 + t + 1) * kT4Keys - 1 > first;
      const int c_at = t % kT4Stages;
      tc_wait(T4_BAR(c_full) + 8 * c_at, (t / kT4Stages) & 1, &s->dead, &g_kv4_status);
      __syncwarp();
      const __half2* par = reinterpret_cast<const __half2*>(smem + kT4OffC + c_at * kT4Stage + 2 * kT4Codes) + tid;
      __half2 k2 = par[0], v2 = par[kT4Keys];
      if (key >= len) k2 = v2 = __float2half2_rn(0.0f);
      const float2 kf = __half22float2(k2), vf = __half22float2(v2);
      const float ks = kf.x * unit, k0 = fmaf(8.0f, kf.x, kf.y) * unit;
      const float w = vf.x, wl = fmaf(8.0f, vf.x, vf.y);
      tc_wait(T4_BAR(s_full) + 8 * p, (t >> 1) & 1, &s->dead, &g_kv4_status);
      __syncwarp();
      tc_fence_after();
      if (lane == 0) tc_arrive(T4_BAR(c_empty) + 8 * c_at);
      uint32_t v[N];
      const uint32_t ts = tmem + 64 * p + lanes, to = tmem + 128 + lanes;
      // v: scores less the running maxima
      auto scores = [&](bool less) {
#pragma unroll
        for (int i = 0; i < N; i += 16) tm_ld16(ts + i, v + i);
        tm_wait_ld();
#pragma unroll
        for (int i = 0; i < N; i += 16) tm_loaded16(v + i);
        const unsigned long long kk = f2pack(ks, ks), cc = f2pack(k0, k0);
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const ulonglong2 qs = *reinterpret_cast<const ulonglong2*>(&s->qsum[i]);
          ulonglong2 ng = make_ulonglong2(0, 0);
          if (less) ng = *reinterpret_cast<const ulonglong2*>(&s->neg[i]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const unsigned long long off = ffma2_to(cc, e ? qs.y : qs.x, e ? ng.y : ng.x);
            const float2 y = f2unpack(ffma2_to(
                kk, f2pack(__uint_as_float(v[i + 2 * e]), __uint_as_float(v[i + 2 * e + 1])), off));
            v[i + 2 * e] = __float_as_uint(y.x);
            v[i + 2 * e + 1] = __float_as_uint(y.y);
          }
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (key > s->lim[i]) v[i] = 0xff800000u;
        }
      };
      scores(true);
      float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < N; i += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          m4[e] = fmaxf(fmaxf(m4[e], __uint_as_float(v[i + e])), __uint_as_float(v[i + e + 4]));
      const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
      if (t4_any(mx > 5.0f || w > vcap)) {
        // larger maxima: of the scores themselves, by warps, then all four
        scores(false);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int x = __float_as_int(fmaxf(__uint_as_float(v[i]), -INFINITY));  // (a NaN is none)
          const int o = __reduce_max_sync(0xffffffffu, x ^ ((x >> 31) & 0x7fffffff));
          if (lane == 0) s->wm[warp][i] = __int_as_float(o ^ ((o >> 31) & 0x7fffffff));
        }
        // of value scales the largest that each query sees: up to this lane's key, then its own
        float vw = fmaxf(w, 0.0f);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const float x = __shfl_up_sync(0xffffffffu, vw, o);
          if (lane >= o) vw = fmaxf(vw, x);
        }
#pragma unroll
        for (int i0 = 0; i0 < N; i0 += 32) {
          const int i = min(i0 + lane, N - 1), last = s->lim[i] - (key - lane);
          const float x = __shfl_sync(0xffffffffu, vw, min(max(last, 0), 31));
          s->wv[warp][i] = last < 0 ? 0.0f : x;
        }
        named_bar_sync(1, 128);
        // the power of two above vm becomes 2^9: weights up to 2^5 stay below 2^15
        auto power = [](float vm, float& cap, float& up) {
          if (!(vm > cap)) return 1.0f;
          const float old = up;
          cap = __uint_as_float(((__float_as_uint(vm) >> 23) + 1) << 23);
          up = 512.0f / cap;
          return up / old;
        };
        auto largest = [&](int i) { return fmaxf(fmaxf(s->wv[0][i], s->wv[1][i]), fmaxf(s->wv[2][i], s->wv[3][i])); };
        if (tid < N) {
          const float mo = s->m[tid];
          const float mn = fmaxf(mo, fmaxf(fmaxf(s->wm[0][tid], s->wm[1][tid]), fmaxf(s->wm[2][tid], s->wm[3][tid])));
          s->m[tid] = mn;
          s->neg[tid] = -mn;
          const float f = mo == -INFINITY ? 0.0f : ex2(mo - mn);
          s->fac[tid] = f;
          s->fo[tid] = f * power(largest(tid), s->cap[tid], s->up[tid]);
        }
        if (!edge) power(largest(0), vcap, vup);
        named_bar_sync(1, 128);
        if (t > 0) {
          tc_wait(T4_BAR(pv_done) + 8 * (p ^ 1), ((t - 1) >> 1) & 1, &s->dead, &g_kv4_status);
          __syncwarp();
          tc_fence_after();
#pragma unroll 1
          for (int k = 0; k < min(t, kT4Sums); ++k)
#pragma unroll 1
            for (int i = 0; i < N; i += 16) {
              uint32_t o[16];
              tm_ld16(to + 64 * k + i, o);
              tm_wait_ld();
              tm_loaded16(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * s->fo[i + e]);
              tm_st16(to + 64 * k + i, o);
            }
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            const unsigned long long f = f2pack(s->fac[2 * i], s->fac[2 * i + 1]);
            asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(l2[i]) : "l"(f));
            asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(z2[i]) : "l"(f));
          }
          tm_wait_st();
        }
        scores(true);
      }
      // weights: to the sums, and times the value's scale to the products
      // (the products of the tile before read the place that these go to)
      if (t > 0) tc_wait(T4_BAR(pv_done) + 8 * (p ^ 1), ((t - 1) >> 1) & 1, &s->dead, &g_kv4_status);
      __syncwarp();
      const float ws = w * vup;
      const unsigned long long wl2 = f2pack(wl, wl);
      uint8_t* at = smem + kT4OffP + tid * 128;
      auto weights = [&](auto apart) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a0 = __uint_as_float(v[i + 2 * e]), a1 = __uint_as_float(v[i + 2 * e + 1]);
            const float x0 = ex2(a0), x1 = ex2(a1);
            const unsigned long long pr = f2pack(x0, x1);
            const int j = i / 2 + e;
            l2[j] = fadd2(l2[j], pr);
            if constexpr (apart.value) {
              const bool s0 = a0 != -INFINITY, s1 = a1 != -INFINITY;
              z2[j] = ffma2_to(pr, f2pack(s0 ? wl : 0.0f, s1 ? wl : 0.0f), z2[j]);
              h[e] = pack_f16x2(s0 ? x0 * (w * s->up[2 * j]) : 0.0f, s1 ? x1 * (w * s->up[2 * j + 1]) : 0.0f);
            } else {
              z2[j] = ffma2_to(pr, wl2, z2[j]);
              h[e] = pack_f16x2(x0 * ws, x1 * ws);
            }
          }
          *reinterpret_cast<uint4*>(at + (((i >> 3) ^ (tid & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
      };
      // (a row that one query sees and another does not may hold a NaN)
      if (edge)
        weights(std::true_type{});
      else
        weights(std::false_type{});
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_arrive(T4_BAR(p_ready) + 8 * p);
    }
    // ---- sums over the keys' threads, then rows of results, through shared memory
    float* part = a.part + (((int64_t)bh * a.nsplit + split) * a.Q + q0) * kK4Rec;
    const bool join = a.nsplit > 1;
    if (n > 0) {
      // (all products are done: the operands' room is free)
      tc_wait(T4_BAR(pv_done) + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, &s->dead, &g_kv4_status);
      __syncwarp();
      tc_fence_after();
      float* red = reinterpret_cast<float*>(smem);               // [2 N][129]
      float* rows = reinterpret_cast<float*>(smem + kT4OffV);    // [N][129]
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float2 x = f2unpack(l2[i]), y = f2unpack(z2[i]);
        red[(2 * i) * 129 + tid] = x.x;
        red[(2 * i + 1) * 129 + tid] = x.y;
        red[(N + 2 * i) * 129 + tid] = y.x;
        red[(N + 2 * i + 1) * 129 + tid] = y.y;
      }
      const int d = 16 * (tid & 7) + (tid >> 3);  // this TMEM lane's dimension
#pragma unroll
      for (int i = 0; i < N; i += 16) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.0f;
#pragma unroll 1
        for (int k = 0; k < min(n, kT4Sums); ++k) {
          uint32_t o[16];
          tm_ld16(tmem + 128 + 64 * k + lanes + i, o);
          tm_wait_ld();
          tm_loaded16(o);
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] += __uint_as_float(o[e]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) rows[(i + e) * 129 + d] = x[e] * (s->cap[i + e] * (1.0f / 512.0f));
      }
      tc_fence_before();
      named_bar_sync(1, 128);
      if (tid < 2 * N) {
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < 128; j += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] += red[tid * 129 + j + e];
        s->total[tid / N][tid % N] = (x[0] + x[1]) + (x[2] + x[3]);
      }
      named_bar_sync(1, 128);
      for (int i = 0; i < nq; ++i) {
        const float L = s->total[0][i], x = rows[i * 129 + tid] + s->total[1][i];
        if (join) {
          part[i * kK4Rec + 4 + tid] = x;
          if (tid == 0) {
            // (natural units, as attention_combine_kernel has them, which takes sums above
            // zero only: where weights are NaN, and so x is, the record has to count)
            part[i * kK4Rec] = isnan(L) ? 0.0f : s->m[i] * 0.6931471805599453f;
            part[i * kK4Rec + 1] = isnan(L) ? 1.0f : L;
          }
        } else {
          const int q = q0 + i, hg = q / T, tok = q - hg * T;
          a.out[(((int64_t)b * T + tok) * a.Hq + kvh * a.G + hg) * kHeadDim + tid] =
              __float2half_rn(L == 0.0f ? 0.0f : x / L);
        }
      }
    } else {
      for (int i = 0; i < nq; ++i) {
        const int q = q0 + i, hg = q / T, tok = q - hg * T;
        if (!join)
          a.out[(((int64_t)b * T + tok) * a.Hq + kvh * a.G + hg) * kHeadDim + tid] = __float2half_rn(0.0f);
        else if (tid < 2)
          part[i * kK4Rec + tid] = tid ? 0.0f : -INFINITY;
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 12)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}
#undef T4_BAR

// CTAs a group of queries: such a number of rounds over the SMs that a CTA's tiles
// and what it costs besides (about twelve) are over soonest (16 x 5 tokens behind
// 30000, 28 / 4 heads: two CTAs a head in one round 154 us, seven in three 168).
static int64_t t4_shares(int64_t groups, int64_t max_ctx) {
  const int64_t tiles = (max_ctx + kT4Keys - 1) / kT4Keys, sms = device_sm_count();
  int64_t best = 1, cost = INT64_MAX;
  for (int64_t S = (tiles + kT4MaxTiles - 1) / kT4MaxTiles; S <= tiles && S <= 64; ++S) {
    const int64_t c = (groups * S + sms - 1) / sms * ((tiles + S - 1) / S + 12) + (S > 1 ? 4 : 0);
    if (c < cost) {
      cost = c;
      best = S;
    }
  }
  return best;
}
static int64_t t4_groups(int64_t Q) { return (Q + kT4Max - 1) / kT4Max; }

template <int N>
static cudaError_t launch_kv4_tc(KV4AttnArgs a, int Z, cudaStream_t st) {
  static std::mutex mu;
  static bool ready[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!ready[dev]) {
      e = cudaFuncSetAttribute(attention_kv4_tc_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, kT4Smem);
      if (e != cudaSuccess) return e;
      ready[dev] = true;
    }
  }
  a.nsplit = (int)t4_shares((int64_t)a.B * a.Hkv * t4_groups(a.Q), a.max_ctx);
  a.cluster = 0;
  e = launch_pdl(attention_kv4_tc_kernel<N>, dim3((unsigned)(a.nsplit * a.B * a.Hkv), (unsigned)Z),
                 dim3(kT4Threads), (size_t)kT4Smem, st, a);
  if (e != cudaSuccess || a.nsplit == 1) return e;
  return launch_attention_combine(a.part, a.B, a.T, a.Hq, a.Hkv, a.nsplit, a.out, st);
}

constexpr int kK4MaxCluster = 16;
constexpr int kK4PerSm = 3;

// How many clusters of S CTAs are resident at once (cached per device).
template <int R>
static cudaError_t k4_resident(int S, int* n) {
  auto k = attention_kv4_kernel<R>;
  static std::mutex mu;
  static bool ready[64] = {false};
  static int cache[64][kK4MaxCluster + 1] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!ready[dev]) {
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, K4Cfg<R>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    ready[dev] = true;
  }
  if (cache[dev][S] == 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)S);
    cfg.blockDim = dim3(kK4Threads);
    cfg.dynamicSmemBytes = K4Cfg<R>::kSmem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int c = 0;
    if (cudaOccupancyMaxActiveClusters(&c, k, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      c = 0;
    }
    cache[dev][S] = c + 1;
  }
  *n = cache[dev][S] - 1;
  return cudaSuccess;
}

static int k4_rows(int64_t Q) { return Q <= 8 ? 1 : 2; }
// Which of the two kernels for more than eight queries: tcgen05 where a code would be
// converted twice or more (Q > 16) and there is work for its longer chain.  28 / 4
// heads, five tokens, us here and in attention_kv4_kernel<2>: one sequence of 2000
// 16.1, 13.7, of 8000 20.5, 21.5, of 30000 28.9, 31.3; 16 of 500 18.9, 17.4, of 2000
// 26.3, 31.5, of 30000 155, 282.  Up to sixteen queries (40 / 8 heads, three tokens,
// 16 of 30000: 250, 193) the other one needs its products once.
static bool k4_long(int64_t heads, int64_t Q, int64_t max_ctx) {
  return Q > 16 && heads * ((Q + 15) / 16) * max_ctx >= 100000;
}

// CTAs that share the keys of a group of queries: as many as fill the SMs, at
// least a step of 32 keys for each of a CTA's warps, and at most kK4MaxSteps:
// mma.sync cuts off what it adds to a sum where an fp32 addition rounds, and the
// codes' part of the values does not cancel as the values do.  1024 steps in one
// sum (64 sequences of 131072, 40 / 8 heads) were off by 1.2e-3 of the result;
// 96 are as many products as attention_kv4_tc_kernel adds up.
constexpr int kK4MaxSteps = 96;
static int64_t k4_least(int64_t max_ctx) {
  constexpr int64_t keys = (int64_t)kK4MaxSteps * kK4Warps * kK4Keys;
  return (max_ctx + keys - 1) / keys;
}
static int64_t k4_shares(int64_t groups, int64_t max_ctx) {
  const int64_t steps = (max_ctx + kK4Keys - 1) / kK4Keys;
  int64_t S = kK4PerSm * (int64_t)device_sm_count() / groups;
  if (S > (steps + kK4Warps - 1) / kK4Warps) S = (steps + kK4Warps - 1) / kK4Warps;
  return std::max(S, k4_least(max_ctx));
}

size_t attention_kv4_workspace_bytes(int B, int T, int Hq, int Hkv, int64_t max_ctx) {
  const int64_t Q = (int64_t)(Hq / Hkv) * T, kq = 8 * k4_rows(Q), groups = (int64_t)B * Hkv * ((Q + kq - 1) / kq);
  const int64_t heads = (int64_t)B * Hkv;
  const int64_t S = !groups                       ? 1
                    : k4_long(heads, Q, max_ctx) ? t4_shares(heads * t4_groups(Q), max_ctx)
                                                 : k4_shares(groups, max_ctx);
  return (S > 1 ? (size_t)(B * (int64_t)Hkv * S * Q) * kK4Rec * sizeof(float) : 0) + 16;
}

// Up to 16 shares meet in a cluster (one launch) as long as all clusters are
// resident; a long cache under few heads takes more, which meet through the
// workspace and a second launch, from eight steps a warp on, and so do those of
// many long caches (k4_least).
template <int R>
static cudaError_t launch_kv4_inst(KV4AttnArgs a, cudaStream_t st) {
  const int Z = (a.Q + 8 * R - 1) / (8 * R);
  const int64_t groups = (int64_t)a.B * a.Hkv * Z;
  int64_t S = k4_shares(groups, a.max_ctx);
  a.cluster = S > 1 && (S <= kK4MaxCluster || a.max_ctx <= (int64_t)kK4MaxCluster * kK4Warps * kK4Keys * 8);
  int n = 0;
  cudaError_t e = k4_resident<R>(1, &n);
  if (e != cudaSuccess) return e;
  if (a.cluster) {
    if (S > kK4MaxCluster) S = kK4MaxCluster;
    for (; S > 1; --S) {
      e = k4_resident<R>((int)S, &n);
      if (e != cudaSuccess) return e;
      if (n >= groups) break;
    }
    a.cluster = S > 1;
    if (S < k4_least(a.max_ctx)) {  // not that many at once: through the workspace
      S = k4_least(a.max_ctx);
      a.cluster = 0;
    }
  }
  a.nsplit = (int)S;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(S * a.B * a.Hkv), (unsigned)Z);
  cfg.blockDim = dim3(kK4Threads);
  cfg.dynamicSmemBytes = K4Cfg<R>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int na = 0;
  if (a.cluster) {
    at[na].id = cudaLaunchAttributeClusterDimension;
    at[na].val.clusterDim.x = (unsigned)S;
    at[na].val.clusterDim.y = at[na].val.clusterDim.z = 1;
    ++na;
  }
  const bool legacy = (st == nullptr || st == cudaStreamLegacy || st == cudaStreamPerThread);
  if (!legacy && pdl_enabled()) {
    at[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[na].val.programmaticStreamSerializationAllowed = 1;
    ++na;
  }
  cfg.attrs = at;
  cfg.numAttrs = na;
  e = cudaLaunchKernelEx(&cfg, attention_kv4_kernel<R>, a);
  if (e != cudaSuccess || a.cluster || S == 1) return e;
  return launch_attention_combine(a.part, a.B, a.T, a.Hq, a.Hkv, a.nsplit, a.out, st);
}

cudaError_t launch_attention_kv4(const __half* qkv, int B, int T, int Hq, int Hkv, const int32_t* pos0,
                                 double theta, const KV4Cache& c, int64_t max_ctx, __half* out, void* ws,
                                 cudaStream_t st) {
  KV4AttnArgs a = {};
  a.qkv = qkv;
  a.c = c;
  a.pos0 = pos0;
  a.out = out;
  a.part = reinterpret_cast<float*>(ws);
  a.B = B;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.Q = a.G * T;
  a.max_ctx = max_ctx;
  a.rf = rope_freq(theta);
  if (k4_long((int64_t)B * Hkv, a.Q, max_ctx)) {
    const int Z = (int)t4_groups(a.Q), n = (a.Q + Z - 1) / Z;
    return n <= 32 ? launch_kv4_tc<32>(a, (a.Q + 31) / 32, st) : launch_kv4_tc<48>(a, Z, st);
  }
  return k4_rows(a.Q) == 1 ? launch_kv4_inst<1>(a, st) : launch_kv4_inst<2>(a, st);
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
