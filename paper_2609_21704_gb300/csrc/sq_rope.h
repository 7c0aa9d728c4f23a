// sq_rope.h -- the rotary embedding, rounded to fp16 once.
//
// A key that goes into four bits is compared with borders between codes, and a
// row's smallest and largest values set its scale: a rotation in plain fp32
// rounds one key value in 5000 to the other fp16 neighbour, and with it now and
// then a whole row of codes.  Here the cosine and sine are pairs of fp32 values
// (head + tail, within 2^-33 of the value: Taylor polynomials on [-pi/4, pi/4],
// the terms that matter in pairs; 2^-34.3 was the worst of six million angles up to
// position 131072), and the rotated value is rounded once: to the nearest fp16 value
// unless it lies within 2^-33 (|a| + |b|) of the middle between two, as about one in
// two million does.  About
// 90 fp32 operations for a position's pair and 10 for most rotated values (30
// for all of them: a packed 4-bit append of 5500 rows took 34 us, not 20); a
// token's table is shared by its heads.  Host code too, so that it can be
// checked against wider arithmetic without a GPU.
#pragma once

#include <math.h>
#include <stdint.h>
#include <string.h>

#ifdef __CUDACC__
#include <cuda_fp16.h>
#define SQ_HD __host__ __device__ __forceinline__
#else
#define SQ_HD inline
#endif

namespace sq {

constexpr int kHeadDim = 128;

// Inverse frequencies theta^(-2d/D), d < D/2, as turns per position in units
// of 2^-64 of a turn: pos * f modulo 2^64 is the angle modulo 2 pi without
// any fp64 arithmetic (two fp64 operations per clock and SM on this GPU: the
// T positions' table cost 2 us per CTA at T = 28).  f comes from fp64, so
// positions up to 2^17 keep the angle within 1e-10, as an fp64 reduction would.
struct RopeFreq {
  unsigned long long f[kHeadDim / 2];
};

// A product rounded by itself (never contracted into a sum behind it).
SQ_HD float mul_rn(float a, float b) {
#ifdef __CUDA_ARCH__
  return __fmul_rn(a, b);
#else
  return a * b;
#endif
}

struct F2 {  // head + tail
  float h, t;
};

SQ_HD F2 f2_mul(F2 a, F2 b) {
  const float p = mul_rn(a.h, b.h);
  const float e = fmaf(a.h, b.h, -p);
  return {p, e + fmaf(a.h, b.t, a.t * b.h)};
}
// a + b for |a| >= |b|
SQ_HD F2 f2_add(F2 a, F2 b) {
  const float s = a.h + b.h;
  const float e = b.h - (s - a.h);
  return {s, e + (a.t + b.t)};
}
SQ_HD F2 f2_norm(F2 a) {
  const float s = a.h + a.t;
  return {s, a.t - (s - a.h)};
}

struct RopeCS {
  F2 c, s;
};

// cos and sin of pos * f (a fraction of a turn in units of 2^-64).
SQ_HD RopeCS rope_cs_pair(int pos, unsigned long long f) {
  const unsigned long long turn = (unsigned long long)(long long)pos * f;
  const unsigned int quad = (unsigned int)((turn + (1ull << 61)) >> 62);  // nearest quarter turn
  const long long r = (long long)(turn - ((unsigned long long)quad << 62));
  const float rh = (float)r;                   // |r| <= 2^61
  const float rl = (float)(r - (long long)rh);
  // times 2 pi 2^-64 (head, tail)
  const float ph = 0x1.921fb6p-62f, pt = -0x1.777a5cp-87f;
  F2 x;
  x.h = mul_rn(rh, ph);
  x.t = fmaf(rh, ph, -x.h) + fmaf(rh, pt, rl * ph);
  x = f2_norm(x);
  const F2 u = f2_norm(f2_mul(x, x));
  // cos x = 1 + u (-1/2 + u (1/24 + u c(u)))
  const float c = fmaf(u.h, fmaf(u.h, fmaf(u.h, 1.0f / 479001600.0f, -1.0f / 3628800.0f), 1.0f / 40320.0f),
                       -1.0f / 720.0f);
  F2 a = f2_add(F2{0x1.555556p-5f, -0x1.555556p-30f}, F2{u.h * c, 0.0f});  // 1/24
  a = f2_add(F2{-0.5f, 0.0f}, f2_mul(u, f2_norm(a)));
  const F2 cx = f2_norm(f2_add(F2{1.0f, 0.0f}, f2_mul(u, f2_norm(a))));
  // sin x = x (1 + u (-1/6 + u (1/120 + u s(u))))
  const float s = fmaf(u.h, fmaf(u.h, -1.0f / 39916800.0f, 1.0f / 362880.0f), -1.0f / 5040.0f);
  F2 b = f2_add(F2{0x1.111112p-7f, -0x1.dddddep-32f}, F2{u.h * s, 0.0f});  // 1/120
  b = f2_add(F2{-0x1.555556p-3f, 0x1.555556p-28f}, f2_mul(u, f2_norm(b)));  // -1/6
  b = f2_add(F2{1.0f, 0.0f}, f2_mul(u, f2_norm(b)));
  const F2 sx = f2_norm(f2_mul(x, f2_norm(b)));
  const F2 nc = {-cx.h, -cx.t}, ns = {-sx.h, -sx.t};
  switch (quad & 3u) {
    case 0: return {cx, sx};
    case 1: return {ns, cx};
    case 2: return {nc, ns};
    default: return {sx, nc};
  }
}

// The fp32 value that rounds to fp16 as a * c + b * s does (a, b fp16 values):
// the sum in a head and a tail, cut to fp32 with its last bit set where
// anything was cut off (fp16 keeps 13 bits fewer, so the second rounding sees
// on which side of a midpoint the sum lies).
SQ_HD float rope_dot(float a, F2 c, float b, F2 s) {
  const float p = mul_rn(a, c.h), q = mul_rn(b, s.h);
  const float sum = p + q;
  const float bb = sum - p;
  const float e = (p - (sum - bb)) + (q - bb);
  const float low = e + (fmaf(a, c.h, -p) + fmaf(b, s.h, -q)) + fmaf(a, c.t, b * s.t);
  float h = sum + low;
  const float t = low - (h - sum);
  if (!(fabsf(h) < INFINITY)) return sum;  // not finite: as plain arithmetic has it
  if (t != 0.0f && h != 0.0f) {
    uint32_t w;
#ifdef __CUDA_ARCH__
    w = __float_as_uint(h);
#else
    memcpy(&w, &h, 4);
#endif
    if ((t < 0.0f) != (h < 0.0f)) w -= 1;  // the sum lies nearer to zero than its head
    w |= 1u;
#ifdef __CUDA_ARCH__
    h = __uint_as_float(w);
#else
    memcpy(&h, &w, 4);
#endif
  }
  return h;
}

#ifdef __CUDACC__
// a * c + b * s rounded to fp16 once.  Plain fp32 is within 2^-22 (|a| + |b|):
// where both ends of 2^-21 round alike, that is the result (all but one value
// in a few hundred).
__device__ __forceinline__ __half rope_f16(float a, F2 c, float b, F2 s) {
  const float v = fmaf(a, c.h, __fmul_rn(b, s.h)), err = (fabsf(a) + fabsf(b)) * 0x1p-21f;
  uint32_t two;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(two) : "f"(v + err), "f"(v - err));
  if ((two >> 16) == (two & 0xffffu)) return __ushort_as_half((uint16_t)two);
  return __float2half_rn(rope_dot(a, c, b, s));
}
#endif

}  // namespace sq
