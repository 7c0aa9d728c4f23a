// sq_logprobs.cu -- log probabilities of given tokens, entropies and top
// alternatives from rows of fp16 logits.
//
//   x_v = (z_v - max z) / T,  S = sum_v e^x_v
//   log p_v = x_v - log S,  H = log S - sum_v e^x_v x_v / S
//
// One reading of the logits: a warp keeps a running maximum and sums relative to
// it, rescaled in the few steps where it grows.  A CTA takes a row, or a cluster
// a row where rows are few; its warps' sums and the maxima of groups of threads
// meet at the end.  Of the entries only those at least the top-th largest of the
// groups' maxima can be among the `top` largest: threads that met one in a
// sixteenth of their part read that again (out of L2), and what passes, some tens
// of entries, is ranked by counting.
// Bound: instructions for many rows, 14 an entry, of which the steps written here need
// about six (1000 rows of 152064, five alternatives: 83 us, 3.7 TB/s, issue 72 % busy);
// for one row the chain of its cluster's three meetings (151936 entries: 7.6 us, 10.4
// with five alternatives).
#include "sq_serve.h"

#include <mutex>

namespace sq {

static __device__ unsigned int g_lp_status;

constexpr int kLpThreads = 256, kLpWarps = kLpThreads / 32;
constexpr int kLpPerSm = 4;       // CTAs that share an SM
constexpr int kLpMaxCluster = 16;
constexpr int kLpList = 512;      // candidates of a CTA
constexpr int kLpSegments = 16;   // parts of a thread's words whose maxima are kept
constexpr int kLpAhead = 4;       // words of a thread in flight

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

// Sums of part of a row relative to its maximum m (a logit's value, at least the
// lowest finite one): of 2^y and y 2^y over entries below it, y = (z - m) c, and
// the number of entries equal to it.
struct LpSums {
  float m, S, E;
  unsigned int eq;
};

struct LpShared {
  uint4 ring[kLpAhead][kLpThreads];  // a thread's words, its own place each
  unsigned long long list[kLpList];  // candidates
  unsigned long long merge[kLpMaxCluster * kLogprobsMaxTop];  // first CTA: every CTA's largest
  uint4 group4[kLpMaxCluster * 8 / 4];  // maxima of the groups of threads of all CTAs
  uint16_t segment[kLpSegments][kLpThreads];  // maxima (in order) of parts of a thread's words
  uint32_t hist[256];
  LpSums warp[kLpWarps];
  LpSums cta[kLpMaxCluster];         // first CTA: of every CTA
  unsigned int over[kLpMaxCluster];  // a CTA's list was too short
  unsigned int count, tau, above, equal;
};

// Joins b's sums to a's; c = log2(e) / T.
__device__ __forceinline__ void lp_join(LpSums& a, const LpSums& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float da = (a.m - m) * c, db = (b.m - m) * c;
  const float fa = lp_ex2(da), fb = lp_ex2(db);
  // entries equal to the lower maximum become ordinary ones
  const float Sa = a.S + (a.m < m ? (float)a.eq : 0.0f), Sb = b.S + (b.m < m ? (float)b.eq : 0.0f);
  a.E = (fa > 0.0f ? fa * fmaf(da, Sa, a.E) : 0.0f) + (fb > 0.0f ? fb * fmaf(db, Sb, b.E) : 0.0f);
  a.S = fmaf(fa, Sa, fb * Sb);
  a.eq = (a.m < m ? 0u : a.eq) + (b.m < m ? 0u : b.eq);
  a.m = m;
}

__device__ __forceinline__ uint32_t lp_word_max(const uint4& q) {
  const __half2* h = reinterpret_cast<const __half2*>(&q);
  const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  const uint32_t b = *reinterpret_cast<const uint32_t*>(&m);
  return max(lp_order16(b & 0xffffu), lp_order16(b >> 16));
}

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

// S CTAs (a cluster) a row.
__global__ void __launch_bounds__(kLpThreads, kLpPerSm) logprobs_kernel(const LogprobArgs a, int S, int groups) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ LpShared s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = S > 1 ? lp_rank() : 0u;
  const int64_t r = blockIdx.x / (unsigned)S;
  const int64_t c0 = a.V * rank / S, c1 = a.V * (rank + 1) / S;
  const int n = (int)(c1 - c0), top = a.top;
  if (tid == 0) s.count = 0;
  __syncwarp();
  if (S > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  // this share in words of eight entries at 16-byte borders; entry i of the
  // share is entry shift + i of the words, and step i of this thread its word
  // i * kLpThreads + tid
  const __half* src = a.z + r * a.V + c0;
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) & 15) >> 1);
  const uint4* data = reinterpret_cast<const uint4*>(src - shift);
  const int words = (n + shift + 7) / 8, steps = (words + kLpThreads - 1) / kLpThreads;
  const int per_segment = (steps + kLpSegments - 1) / kLpSegments;
  // this warp's steps of whole words only: plain0 <= i < plain1
  const int plain0 = shift > 0 && warp == 0 ? 1 : 0;
  const int plain1 = ((n + shift) / 8 - warp * 32 - 32 + kLpThreads) / kLpThreads;
  auto whole = [&](int w) { return w * 8 >= shift && w * 8 + 8 <= n + shift; };
  // a word; at the ends entry by entry, -inf for what is not in the share
  auto load = [&](int w) {
    if (whole(w)) return __ldg(data + w);
    uint4 q = make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u);
    uint16_t* h = reinterpret_cast<uint16_t*>(&q);
    if (w < words)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (w * 8 + i >= shift && w * 8 + i < n + shift) h[i] = __half_as_ushort(src[w * 8 + i - shift]);
    return q;
  };

  // ---- the walk.  y = z c + b, b = -m c rounded once for the warp's maximum m
  // (what that is off by is put right at the end); entries equal to m are counted
  // and left out of the sums, so that what lies beside a sure token is kept.  An
  // entry of -inf makes the second sum NaN (0 x -inf): the warp then walks again
  // with y cut off at -150, where 2^y is zero.
  const float c = a.invT * 1.4426950408889634f;
  uint32_t mine = 0;  // this thread's maximum, in order
  LpSums sum;
#pragma unroll 1
  for (int cut = 0; cut < 2; ++cut) {
    unsigned long long Sa = 0, Sb = 0, Ea = 0, Eb = 0;
    const unsigned long long c2 = f2pack(c, c);
    uint32_t mo = lp_order16(0xfbffu), seg = 0;
    __half2 mh2 = __half2half2(__ushort_as_half(0xfbff));
    __half2 mx = __half2half2(__ushort_as_half(0xfc00));
    float m = -65504.0f, b = 65504.0f * c;
    unsigned int eq = 0;
    const uint32_t ring = smem_u32(&s.ring[0][tid]);
    auto request = [&](int i) {
      if (i >= plain0 && i < plain1)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                         ring + (uint32_t)(i % kLpAhead) * (uint32_t)(kLpThreads * 16)),
                     "l"(data + i * kLpThreads + tid)
                     : "memory");
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kLpAhead - 1; ++i) request(i);
    int left = per_segment;
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
      request(i + kLpAhead - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kLpAhead - 1) : "memory");
      const bool plain = i >= plain0 && i < plain1;
      uint4 q = s.ring[i % kLpAhead][tid];
      if (!plain) q = load(i * kLpThreads + tid);
      const __half2* h = reinterpret_cast<const __half2*>(&q);
      const __half2 wm = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
      mx = __hmax2_nan(mx, wm);
      const bool grown = !__hblt2(wm, mh2);  // (a NaN is not less either)
      const unsigned long long b2 = f2pack(b, b);
      float y[8], e[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 x = __half22float2(h[k]);
        unsigned long long yy;
        asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(yy) : "l"(f2pack(x.x, x.y)), "l"(c2), "l"(b2));
        const float2 v = f2unpack(yy);
        y[2 * k] = v.x;
        y[2 * k + 1] = v.y;
        e[2 * k] = lp_ex2(v.x);
        e[2 * k + 1] = lp_ex2(v.y);
      }
      if (__any_sync(0xffffffffu, grown) || !plain || cut) {
        const uint32_t o = __reduce_max_sync(0xffffffffu, lp_word_max(q));
        if (o > mo) {  // a larger maximum: the sums relative to it
          mo = o;
          const float m1 = lp_value(o), b1 = __fmul_rn(-m1, c), d = b1 - b, f = lp_ex2(d);
          const float2 s0 = f2unpack(Sa), s1 = f2unpack(Sb), e0 = f2unpack(Ea), e1 = f2unpack(Eb);
          const float S0 = (s0.x + s0.y) + (s1.x + s1.y) + (float)eq, E0 = (e0.x + e0.y) + (e1.x + e1.y);
          Sa = f2pack(f * S0, 0.0f);
          Ea = f2pack(f > 0.0f ? f * fmaf(d, S0, E0) : 0.0f, 0.0f);
          Sb = Eb = 0;
          eq = 0;
          m = m1;
          b = b1;
          mh2 = __half2half2(__float2half_rn(m1));
        }
        const uint16_t* z = reinterpret_cast<const uint16_t*>(&q);
        const int w = i * kLpThreads + tid;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const bool in = w * 8 + k >= shift && w * 8 + k < n + shift;
          const bool one = in && lp_order16(z[k]) == mo;
          eq += one;
          float v = fmaf(__half2float(__ushort_as_half(z[k])), c, b);
          if (cut || !in) v = fmaxf(v, -150.0f);
          y[k] = v;
          e[k] = one || !in ? 0.0f : lp_ex2(v);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        const unsigned long long ea = f2pack(e[2 * k], e[2 * k + 1]), eb = f2pack(e[2 * k + 2], e[2 * k + 3]);
        asm("add.rn.f32x2 %0, %0, %1;" : "+l"(Sa) : "l"(ea));
        asm("add.rn.f32x2 %0, %0, %1;" : "+l"(Sb) : "l"(eb));
        ffma2(Ea, ea, f2pack(y[2 * k], y[2 * k + 1]));
        ffma2(Eb, eb, f2pack(y[2 * k + 2], y[2 * k + 3]));
      }
      if (--left == 0 || i == steps - 1) {
        const uint32_t bits = *reinterpret_cast<const uint32_t*>(&mx);
        const uint32_t o = max(lp_order16(bits & 0xffffu), lp_order16(bits >> 16));
        s.segment[seg++][tid] = (uint16_t)o;
        mine = max(mine, o);
        mx = __half2half2(__ushort_as_half(0xfc00));
        left = per_segment;
      }
    }
    const float2 s0 = f2unpack(Sa), s1 = f2unpack(Sb), e0 = f2unpack(Ea), e1 = f2unpack(Eb);
    sum.m = m;
    sum.S = warp_sum((s0.x + s0.y) + (s1.x + s1.y));
    sum.E = warp_sum((e0.x + e0.y) + (e1.x + e1.y));
    sum.eq = __reduce_add_sync(0xffffffffu, eq);
    // y is `skew` less than (z - m) c.  At a small temperature it is large (m c may
    // be 10^35, rounded), and no entry but the largest has any weight: nothing to put right.
    if (sum.S > 0.0f) {
      const float skew = fmaf(-m, c, -b), f = lp_ex2(skew);
      sum.E = f * fmaf(skew, sum.S, sum.E);
      sum.S *= f;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!isnan(sum.E)) break;  // (the whole warp)
  }

  // ---- the groups' maxima to every CTA of the row, sums to the first
  uint32_t* group = reinterpret_cast<uint32_t*>(s.group4);
  const int total = S * groups;  // 32 to 128
  __syncwarp();
  if (S > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // all have begun
  {
    uint32_t o = mine;
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
  if (lane == 0) s.warp[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    // lanes 0 .. 7 a warp's sums each, joined in pairs
    LpSums t = s.warp[lane & 7];
#pragma unroll
    for (int i = 4; i > 0; i >>= 1) {
      LpSums u;
      u.m = __shfl_down_sync(0xffffffffu, t.m, i);
      u.S = __shfl_down_sync(0xffffffffu, t.S, i);
      u.E = __shfl_down_sync(0xffffffffu, t.E, i);
      u.eq = __shfl_down_sync(0xffffffffu, t.eq, i);
      lp_join(t, u, c);
    }
    if (lane == 0) {
      if (S > 1) {
        lp_st32(&s.cta[rank].m, 0u, __float_as_uint(t.m));
        lp_st32(&s.cta[rank].S, 0u, __float_as_uint(t.S));
        lp_st32(&s.cta[rank].E, 0u, __float_as_uint(t.E));
        lp_st32(&s.cta[rank].eq, 0u, t.eq);
      } else {
        s.cta[0] = t;
      }
    }
  }
  lp_sync(S);
  if (tid < total) {
    const uint32_t key = group[tid];
    int above = 0;
#pragma unroll 4
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

  // the given token's logit, on its way while candidates are collected
  const bool answers = rank == 0 && tid == 0;
  float zt = 0.0f;
  bool token_ok = false;
  if (answers && a.tokens) {
    const int64_t t = a.tokens[r];
    token_ok = t >= 0 && t < a.V;
    if (token_ok) zt = __half2float(a.z[r * a.V + t]);
  }
  if (top > 0) {
    uint32_t tau = s.tau;
    unsigned int ties = 0;  // this warp's entries equal to tau so far
    // Candidates: entries above tau, and of those equal to it the first `top` of
    // a warp, whose words are taken in rising order.
    auto collect = [&]() {
      const int segments = (steps + per_segment - 1) / per_segment;
#pragma unroll 1
      for (int g = 0; g < segments; ++g) {
        const bool look = s.segment[g][tid] >= tau;
        if (!__any_sync(0xffffffffu, look)) continue;
        const int i1 = min((g + 1) * per_segment, steps);
#pragma unroll 1
        for (int i0 = g * per_segment; i0 < i1; i0 += 4) {
          uint4 qs[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            qs[k] = make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u);
            if (look && i0 + k < i1) qs[k] = load((i0 + k) * kLpThreads + tid);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int w = (i0 + k) * kLpThreads + tid;
            const bool any = look && i0 + k < i1 && lp_word_max(qs[k]) >= tau;
            if (!__any_sync(0xffffffffu, any)) continue;
            const uint16_t* z = reinterpret_cast<const uint16_t*>(&qs[k]);
            uint32_t here = 0;  // bits: ties, and above them entries over tau
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t o = lp_order16(z[e]);
              const bool in = any && w * 8 + e >= shift && w * 8 + e < n + shift;
              here |= (in && o == tau ? 1u : 0u) << e | (in && o > tau ? 256u : 0u) << e;
            }
            unsigned int before = __popc(here & 255u);  // ties of lower lanes
            const unsigned int own = before;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
              const unsigned int v = __shfl_up_sync(0xffffffffu, before, d);
              if (lane >= d) before += v;
            }
            const unsigned int all = __shfl_sync(0xffffffffu, before, 31);
            before += ties - own;
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
              bool take = (here >> (8 + e)) & 1u;
              if ((here >> e) & 1u) take = before++ < (unsigned)top;
              if (take) {
                const unsigned int at = atomicAdd(&s.count, 1u);
                const int64_t v = w * 8 + e - shift;
                if (at < kLpList)
                  s.list[at] = lp_key(lp_order16(__half_as_ushort(src[v])), (uint32_t)(c0 + v));
              }
            }
            ties += all;
          }
        }
      }
    };
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
#pragma unroll 1
    for (int again = 0; again < 2; ++again) {
      collect();
      __syncthreads();
      if (tid < S) {
        const uint32_t o = s.count > kLpList;
        if (S > 1)
          lp_st32(&s.over[rank], (uint32_t)tid, o);
        else
          s.over[0] = o;
      }
      deliver();
      lp_sync(S);
      bool over = false;
      for (int i = 0; i < S; ++i) over |= s.over[i] != 0;
      if (!over || again) break;
      // Rarely (rows in order, say) more pass than the list holds.  Then tau
      // becomes the top-th largest logit itself, by two walks that count its
      // upper and its lower byte.
      uint32_t prefix = 0;
      unsigned int above = 0;  // entries above the bytes found so far
#pragma unroll 1
      for (int byte = 1; byte >= 0; --byte) {
        lp_sync(S);  // (the others have read the last counts)
        s.hist[tid] = 0;
        __syncthreads();
#pragma unroll 1
        for (int w = tid; w < words; w += kLpThreads) {
          const uint4 q = load(w);
          const uint16_t* z = reinterpret_cast<const uint16_t*>(&q);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t o = lp_order16(z[e]);
            if (w * 8 + e >= shift && w * 8 + e < n + shift && (byte == 1 || (o >> 8) == prefix))
              atomicAdd(&s.hist[byte == 1 ? o >> 8 : o & 255u], 1u);
          }
        }
        lp_sync(S);
        unsigned int cnt = 0;
        for (int i = 0; i < S; ++i) cnt += S > 1 ? lp_ld32(&s.hist[tid], (uint32_t)i) : s.hist[tid];
        __syncthreads();
        s.list[tid] = cnt;
        __syncthreads();
        unsigned int over_me = above;
        for (int j = tid + 1; j < 256; ++j) over_me += (unsigned int)s.list[j];
        if (over_me < (unsigned)top && over_me + cnt >= (unsigned)top) {
          s.tau = byte == 1 ? (uint32_t)tid : (prefix << 8) | (uint32_t)tid;
          s.equal = over_me;
        }
        __syncthreads();
        prefix = s.tau;
        above = s.equal;
      }
      tau = prefix;
      __syncthreads();
      if (tid == 0) s.count = 0;
      ties = 0;
      __syncthreads();
    }
  }
  if (rank == 0) {
    LpSums t = s.cta[0];
    for (int i = 1; i < S; ++i) lp_join(t, s.cta[i], c);
    const float rest = t.S + (float)(t.eq - 1);
    const float lse = log1pf(rest);
    if (answers) {
      if (a.entropy) a.entropy[r] = lse - t.E * 0.6931471805599453f / (1.0f + rest);
      if (a.tokens) {
        if (!token_ok) atomicOr(&g_lp_status, SQ_DEV_BAD_TOKEN_ID);
        a.logprob[r] = token_ok ? (zt - m) * a.invT - lse : NAN;
      }
    }
    if (top > 0)
      lp_ranked(s.merge, S * top, top, [&](int i, unsigned long long key) {
        a.top_tokens[r * top + i] = (int32_t)(0xffffffffu - (uint32_t)key);
        a.top_logprobs[r * top + i] = (lp_value((uint32_t)(key >> 32)) - m) * a.invT - lse;
      });
  }
}

// CTAs a row: one, or as many as fill the SMs (up to 16, in shares of 4096
// entries at least) where rows are few. Above ten alternatives a row has eight
// at most: its first CTA ranks the lists of all of them (one row of 151936, 20
// alternatives: 13.8 us with eight, 15.8 with sixteen; 16 rows 16.0 and 21.2;
// with five alternatives, one row: 11.5 and 10.4).
cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t st) {
  static std::mutex mu;
  static bool ready[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!ready[dev]) {
      e = cudaFuncSetAttribute(logprobs_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      ready[dev] = true;
    }
  }
  int64_t S = (int64_t)kLpPerSm * device_sm_count() / 2 / a.R;
  if (S > a.V / 4096) S = a.V / 4096;
  if (S > kLpMaxCluster) S = kLpMaxCluster;
  if (a.top > 10 && S > 8) S = 8;
  if (S < 1) S = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.R * S));
  cfg.blockDim = dim3(kLpThreads);
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
