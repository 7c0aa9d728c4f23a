// sq_logprobs.cu -- log probabilities of given tokens, entropies and top
// alternatives from rows of fp16 logits.
//
//   x_v = (z_v - max z) / T,  S = sum_v e^x_v
//   log p_v = x_v - log S,  H = log S - sum_v e^x_v x_v / S
//
// A cluster of CTAs takes a row and keeps it in shared memory, so that logits
// are read from memory once although they are walked twice: for the maximum,
// then for the sums.  The entries that may be among the `top` largest are found
// on the second walk without sorting: the top-th largest of the maxima of
// groups of threads bounds them from below, and about one entry in a thousand
// passes.  They are ranked by counting, in each CTA and then in the first.
// Bound: the logits' bytes from memory for many rows; for one row the cluster's
// three meetings.
#include "sq_serve.h"

#include <mutex>

namespace sq {

static __device__ unsigned int g_lp_status;

constexpr int kLpThreads = 256, kLpWarps = kLpThreads / 32;
constexpr int kLpChunk = 25600;    // entries of a CTA, where clusters of 16 allow it
constexpr int kLpMaxCluster = 16;
constexpr int kLpList = 512;       // candidates of a CTA
constexpr int kLpParts = 4;        // copies of a CTA's share, each waited for by itself

// Total order of (logit, index): largest logit first, lowest index among
// equals (-0 equals 0).  Larger keys come first; 0 is no entry's key.
__device__ __forceinline__ uint32_t lp_order16(uint32_t b) {
  if (b == 0x8000u) b = 0;
  return b & 0x8000u ? 0xffffu - b : b | 0x8000u;
}
__device__ __forceinline__ float lp_value(uint32_t order) {
  return __half2float(__ushort_as_half((uint16_t)(order & 0x8000u ? order & 0x7fffu : 0xffffu - order)));
}
__device__ __forceinline__ unsigned long long lp_key(uint32_t order, uint32_t v) {
  return ((unsigned long long)order << 32) | (0xffffffffu - v);
}

__device__ __forceinline__ uint32_t lp_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void lp_sync(int S) {
  __syncwarp();
  if (S > 1)
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else
    __syncthreads();
}
__device__ __forceinline__ uint32_t lp_remote(const void* local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(local)), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t lp_ld32(const void* local, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(lp_remote(local, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void lp_st32(const void* local, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(lp_remote(local, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void lp_st64(const void* local, uint32_t rank, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(lp_remote(local, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct LpShared {
  unsigned long long list[kLpList];  // candidates
  unsigned long long merge[kLpMaxCluster * kLogprobsMaxTop];  // first CTA: every CTA's largest
  uint64_t bar[kLpParts];
  uint4 group4[kLpMaxCluster * 8 / 4];  // maxima of the groups of threads of all CTAs
  uint32_t hist[256];
  float sum[2][kLpWarps];
  float total[2][kLpMaxCluster];     // first CTA: sums of every CTA
  unsigned int ones[kLpMaxCluster];
  unsigned int over[kLpMaxCluster];  // a CTA's list was too short
  unsigned int count, equal, tau, above;
};

// Ranks n keys of the list by counting; the first k go to `best`.
template <typename Emit>
__device__ __forceinline__ void lp_ranked(const unsigned long long* list, int n, int k, Emit emit) {
  for (int i = threadIdx.x; i < n; i += kLpThreads) {
    const unsigned long long key = list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > key;
    if (key && rank < k) emit(rank, key);
  }
}

// S CTAs (a cluster) a row; dynamic shared memory: the share of the row, at
// the same place within 16 bytes as in memory.
__global__ void __launch_bounds__(kLpThreads, 4) logprobs_kernel(const LogprobArgs a, int S, int groups) {
  griddep_wait();
  griddep_launch_dependents();
  extern __shared__ __align__(128) uint8_t lp_smem[];
  __shared__ LpShared s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = S > 1 ? lp_rank() : 0u;
  const int64_t r = blockIdx.x / (unsigned)S;
  const int64_t c0 = a.V * rank / S, c1 = a.V * (rank + 1) / S;
  const int n = (int)(c1 - c0), top = a.top;
  const __half* z = a.z + r * a.V;
  const __half* src = z + c0;
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) & 15) >> 1);  // entries before ours in the first 16 bytes
  const int words = (n + shift + 7) / 8;
  __half* row = reinterpret_cast<__half*>(lp_smem);  // entry i of the share at row[shift + i]

  // ---- the share: whole 16-byte pieces by bulk copies, ragged ends by hand
  const int w0 = shift ? 1 : 0, w1 = max((n + shift) / 8, w0);  // whole words
  if (tid == 0) {
    for (int p = 0; p < kLpParts; ++p) mbar_init(&s.bar[p], 1);
    fence_mbar_init();
    s.count = s.equal = 0;
    for (int p = 0; p < kLpParts; ++p) {
      const int b = w0 + (int)((int64_t)(w1 - w0) * p / kLpParts), e = w0 + (int)((int64_t)(w1 - w0) * (p + 1) / kLpParts);
      mbar_arrive_expect_tx(&s.bar[p], (uint32_t)(e - b) * 16);
      if (e > b) bulk_g2s(lp_smem + b * 16, src - shift + b * 8, (uint32_t)(e - b) * 16, &s.bar[p]);
    }
  }
  // ends, and what pads the first and the last word: -inf
  if (tid < 16) {
    const int i = tid < 8 ? tid : w1 * 8 + tid - 8;  // place in shared memory
    if (tid < 8 ? w0 > 0 : w1 < words)
      row[i] = i >= shift && i < shift + n ? src[i - shift] : __ushort_as_half(0xfc00);
  }
  __syncwarp();
  if (S > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  __syncthreads();

  // ---- first walk: maxima (a NaN stays one)
  __half2 mx = __halves2half2(__ushort_as_half(0xfc00), __ushort_as_half(0xfc00));
  bool late = false;
  {
    int part = 0;
    for (int w = tid; w < words; w += kLpThreads) {
      // every part up to the one that holds this word
      while (part < kLpParts && w >= w0 + (int)((int64_t)(w1 - w0) * part / kLpParts)) {
        late |= !mbar_wait_bounded(&s.bar[part], 0u);
        ++part;
      }
      const uint4 q = reinterpret_cast<const uint4*>(lp_smem)[w];
      const __half2* h = reinterpret_cast<const __half2*>(&q);
      mx = __hmax2_nan(__hmax2_nan(mx, __hmax2_nan(h[0], h[1])), __hmax2_nan(h[2], h[3]));
    }
    for (; part < kLpParts; ++part) late |= !mbar_wait_bounded(&s.bar[part], 0u);
  }
  if (late) atomicOr(&g_lp_status, SQ_DEV_TIMEOUT);
  // ---- the row's maximum, and the top-th largest of the groups' maxima: every
  // CTA gets them all (written to it: a read would wait for the way there too)
  uint32_t* group = reinterpret_cast<uint32_t*>(s.group4);
  const int total = S * groups;  // 32 to 128
  __syncwarp();
  if (S > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // all have begun
  {
    const uint32_t b = *reinterpret_cast<const uint32_t*>(&mx);
    uint32_t o = max(lp_order16(b & 0xffffu), lp_order16(b >> 16));
    const int span = kLpThreads / groups;  // threads of a group: 8, 16 or 32
    for (int i = span >> 1; i > 0; i >>= 1) o = max(o, __shfl_xor_sync(0xffffffffu, o, i));
    const uint32_t at = rank * groups + tid / span;
    o = (o << 8) | (255u - at);  // different keys for equal maxima
    if (S == 1) {
      if (tid % span == 0) group[at] = o;
    } else {
      for (int i = tid % span; i < S; i += span) lp_st32(&group[at], (uint32_t)i, o);
    }
  }
  lp_sync(S);
  if (tid < total) {
    const uint32_t key = group[tid];
    int above = 0;
    for (int j = 0; j < total / 4; ++j) {
      const uint4 q = s.group4[j];
      above += (q.x > key) + (q.y > key) + (q.z > key) + (q.w > key);
    }
    if (above == 0) s.above = key >> 8;
    if (above == (top > 0 ? top - 1 : 0)) s.tau = key >> 8;
  }
  __syncthreads();
  const uint32_t mo = s.above;
  const float m = lp_value(mo);
  const bool bad = mo >= 0xfc00u, none = mo == 0x3ffu;  // +inf or NaN; nothing but -inf
  if (bad || none) {
    if (rank == 0) {
      if (tid == 0) {
        atomicOr(&g_lp_status, bad ? SQ_DEV_NONFINITE_LOGIT : SQ_DEV_NO_MASS);
        if (a.logprob) a.logprob[r] = NAN;
        if (a.entropy) a.entropy[r] = NAN;
      }
      if (tid < top) {
        a.top_tokens[r * top + tid] = -1;
        a.top_logprobs[r * top + tid] = NAN;
      }
    }
    return;  // (nothing more is written to or read from another CTA)
  }

  // Candidates of one word: entries above tau, and of those equal to it the
  // first `top` of a warp, whose words come in rising order.
  unsigned int ties = 0;  // this warp's
  auto offer = [&](const uint16_t* h, int w, bool any, uint32_t tau) {
    if (!__any_sync(0xffffffffu, any)) return;
    unsigned int mine = 0, hits = 0;
    uint32_t o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = w * 8 + e - shift;
      o[e] = any && i >= 0 && i < n ? lp_order16(h[e]) : 0u;
      mine += o[e] == tau;
      hits |= (o[e] > tau ? 1u : 0u) << e;
    }
    unsigned int before = mine;  // ties of lower lanes
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned int v = __shfl_up_sync(0xffffffffu, before, d);
      if (lane >= d) before += v;
    }
    const unsigned int all = __shfl_sync(0xffffffffu, before, 31);
    before -= mine;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bool take = (hits >> e) & 1;
      if (o[e] == tau && o[e]) take = ties + before++ < (unsigned)top;
      if (take) {
        const unsigned int at = atomicAdd(&s.count, 1u);
        if (at < kLpList) s.list[at] = lp_key(o[e], (uint32_t)(c0 + w * 8 + e - shift));
      }
    }
    ties += all;
  };

  // ---- second walk: the sums, apart from entries equal to the maximum (their
  // terms are ones, counted: a sure row's logarithm keeps what is left)
  uint32_t tau = s.tau;
  unsigned int ones = 0;
  {
    const float sc = a.invT * 1.4426950408889634f;
    const unsigned long long m2 = f2pack(-m, -m), sc2 = f2pack(sc, sc);
    unsigned long long Sa = 0, Sb = 0, Ea = 0, Eb = 0;
    const __half2 tau2 = __half2half2(__float2half_rn(lp_value(tau))), mh2 = __half2half2(__float2half_rn(m));
    for (int wb = 0; wb < words; wb += kLpThreads) {
      const int w = wb + tid;
      uint4 q = make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u);
      if (w < words) q = reinterpret_cast<const uint4*>(lp_smem)[w];
      const __half2* h = reinterpret_cast<const __half2*>(&q);
      const __half2 wm = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
      const bool any = w < words && !__hblt2(wm, tau2);  // an entry at tau or above
      const bool near = any && !__hblt2(wm, mh2);        // at the maximum
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = __half22float2(h[e]);
        unsigned long long y;
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(f2pack(f.x, f.y)), "l"(m2));
        asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(y) : "l"(sc2));
        float2 x = f2unpack(y);
        x.x = fmaxf(x.x, -150.0f);  // (-inf: no weight, 2^-150 is zero, and no NaN in the entropy)
        x.y = fmaxf(x.y, -150.0f);
        y = f2pack(x.x, x.y);
        float e0 = lp_ex2(x.x), e1 = lp_ex2(x.y);
        if (near) {
          ones += (f.x == m) + (f.y == m);
          e0 = f.x == m ? 0.0f : e0;
          e1 = f.y == m ? 0.0f : e1;
        }
        const unsigned long long ee = f2pack(e0, e1);
        if (e & 1) {
          asm("add.rn.f32x2 %0, %0, %1;" : "+l"(Sb) : "l"(ee));
          ffma2(Eb, ee, y);
        } else {
          asm("add.rn.f32x2 %0, %0, %1;" : "+l"(Sa) : "l"(ee));
          ffma2(Ea, ee, y);
        }
      }
      if (top > 0) offer(reinterpret_cast<const uint16_t*>(&q), w, any, tau);
    }
    const float2 s0 = f2unpack(Sa), s1 = f2unpack(Sb), e0 = f2unpack(Ea), e1 = f2unpack(Eb);
    const float S0 = warp_sum((s0.x + s0.y) + (s1.x + s1.y)), E0 = warp_sum((e0.x + e0.y) + (e1.x + e1.y));
    ones = __reduce_add_sync(0xffffffffu, ones);
    if (lane == 0) {
      s.sum[0][warp] = S0;
      s.sum[1][warp] = E0;
      if (ones) atomicAdd(&s.equal, ones);
    }
  }
  __syncthreads();
  // results to the first CTA; whether a list was too short to all
  if (tid < 2) {
    float t = 0.0f;
    for (int i = 0; i < kLpWarps; ++i) t += s.sum[tid][i];
    if (S > 1)
      lp_st32(&s.total[tid][rank], 0u, __float_as_uint(t));
    else
      s.total[tid][0] = t;
  } else if (tid == 2) {
    if (S > 1)
      lp_st32(&s.ones[rank], 0u, s.equal);
    else
      s.ones[0] = s.equal;
  } else if (tid >= 32 && tid < 32 + S) {
    const uint32_t o = s.count > kLpList;
    if (S > 1)
      lp_st32(&s.over[rank], (uint32_t)(tid - 32), o);
    else
      s.over[0] = o;
  }
  // this CTA's `top` largest of its list to the first CTA
  auto deliver = [&]() {
    const int have = min((int)s.count, kLpList);
    for (int i = tid + have; i < top; i += kLpThreads)  // places that stay empty
      if (S > 1)
        lp_st64(&s.merge[rank * top + i], 0u, 0ull);
      else
        s.merge[i] = 0;
    lp_ranked(s.list, have, top, [&](int i, unsigned long long key) {
      if (S > 1)
        lp_st64(&s.merge[rank * top + i], 0u, key);
      else
        s.merge[i] = key;
    });
  };
  if (top > 0) deliver();
  lp_sync(S);

  // ---- rarely (rows in order, say) more pass than the list holds: the top-th
  // largest logit itself, by two walks that count its upper and its lower byte
  if (top > 0) {
    bool over = false;
    for (int i = 0; i < S; ++i) over |= s.over[i] != 0;
    if (over) {
      uint32_t prefix = 0;
      unsigned int above = 0;  // entries above the bytes found so far
      for (int byte = 1; byte >= 0; --byte) {
        lp_sync(S);  // (the others have read the last counts)
        s.hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kLpThreads) {
          const uint32_t o = lp_order16(__half_as_ushort(row[shift + i]));
          if (byte == 1 || (o >> 8) == prefix) atomicAdd(&s.hist[byte == 1 ? o >> 8 : o & 255u], 1u);
        }
        lp_sync(S);
        unsigned int c = 0;
        for (int i = 0; i < S; ++i) c += S > 1 ? lp_ld32(&s.hist[tid], (uint32_t)i) : s.hist[tid];
        __syncthreads();
        s.list[tid] = c;
        __syncthreads();
        unsigned int over_me = above;
        for (int j = tid + 1; j < 256; ++j) over_me += (unsigned int)s.list[j];
        if (over_me < (unsigned)top && over_me + c >= (unsigned)top) {
          s.tau = byte == 1 ? (uint32_t)tid : (prefix << 8) | (uint32_t)tid;
          s.above = over_me;
        }
        __syncthreads();
        prefix = s.tau;
        above = s.above;
      }
      tau = prefix;
      if (tid == 0) s.count = 0;
      ties = 0;
      __syncthreads();
      for (int wb = 0; wb < words; wb += kLpThreads) {
        const int w = wb + tid;
        uint4 q = make_uint4(0, 0, 0, 0);
        if (w < words) q = reinterpret_cast<const uint4*>(lp_smem)[w];
        offer(reinterpret_cast<const uint16_t*>(&q), w, w < words, tau);
      }
      __syncthreads();
      deliver();
      lp_sync(S);
    }
  }
  if (rank == 0) {
    float t0 = 0.0f, t1 = 0.0f;
    unsigned int eq = 0;
    for (int i = 0; i < S; ++i) {
      t0 += s.total[0][i];
      t1 += s.total[1][i];
      eq += s.ones[i];
    }
    const float rest = t0 + (float)(eq - 1);
    const float lse = log1pf(rest);
    if (tid == 0) {
      if (a.entropy) a.entropy[r] = lse - t1 * 0.6931471805599453f / (1.0f + rest);
      if (a.tokens) {
        const int64_t t = a.tokens[r];
        const bool ok = t >= 0 && t < a.V;
        if (!ok) atomicOr(&g_lp_status, SQ_DEV_BAD_TOKEN_ID);
        a.logprob[r] = ok ? (__half2float(z[t]) - m) * a.invT - lse : NAN;
      }
    }
    if (top > 0)
      lp_ranked(s.merge, S * top, top, [&](int i, unsigned long long key) {
        a.top_tokens[r * top + i] = (int32_t)(0xffffffffu - (uint32_t)key);
        a.top_logprobs[r * top + i] = (lp_value((uint32_t)(key >> 32)) - m) * a.invT - lse;
      });
  }
}

// CTAs a row: shares of kLpChunk entries; more of them where rows alone leave
// SMs idle, down to shares of 4096.
cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t st) {
  static std::mutex mu;
  static bool ready[64] = {false};
  constexpr int kMaxSmem = 2 * ((1 << 20) / kLpMaxCluster + 16);
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!ready[dev]) {
      e = cudaFuncSetAttribute(logprobs_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(logprobs_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      ready[dev] = true;
    }
  }
  int64_t S = (a.V + kLpChunk - 1) / kLpChunk;
  if (S > kLpMaxCluster) S = kLpMaxCluster;
  while (2 * S <= kLpMaxCluster && 2 * S * a.R <= device_sm_count() && a.V / (2 * S) >= 4096) S *= 2;
  const int64_t share = (a.V + S - 1) / S;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.R * S));
  cfg.blockDim = dim3(kLpThreads);
  cfg.dynamicSmemBytes = (size_t)((share + 15) / 8 * 16);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int na = 0;
  if (S > 1) {
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
  // groups of threads whose maxima are kept: 32 a row at least
  const int groups = S == 1 ? 32 : S < 4 ? 16 : 8;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel, a, (int)S, groups);
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
