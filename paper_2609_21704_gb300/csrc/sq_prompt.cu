// sq_prompt.cu -- attention over whole prompts: packed sequences of different
// lengths, causal, grouped heads, each behind the prefix that its cache holds.
//
//   k'_t = fp16(R(pos_t) k_t), cached with v_t at pos_t = pos0 + t
//   out_t = sum_{j <= pos_t} p_tj v_j / sum_j p_tj,
//   p_tj = exp(q'_t . k'_j / sqrt(D)), q'_t = fp16(R(pos_t) q_t)
// (R by rope_f16 for what is kept, in plain fp32 for queries).
//
// Two launches.  prompt_prepare_kernel rotates and appends, writes the rotated
// queries where TMA can fetch them, and one of its CTAs lays out the work of
// the second launch from the lengths on the device, so that a captured call
// serves other lengths on replay.  prompt_attention_kernel: one persistent CTA
// an SM on tcgen05.
#include "sq_packed.cuh"
#include "sq_tcgen.cuh"

#include <mutex>
#include <stddef.h>

namespace sq {

static __device__ unsigned int g_prompt_status;

constexpr int kPrRows = 256;    // query rows of a work item: two MMA tiles
constexpr int kPrKeys = 128;    // keys of a block
constexpr int kPrTile = kPrKeys * kHeadDim * 2;  // bytes of a block's keys (or values)
constexpr int kPrK = 2, kPrV = 3;  // tiles of keys and of values in shared memory
constexpr int kPrPrepThreads = 256;
constexpr int kPrMaxBlocks = (int)(kPromptMaxCtx / kPrKeys);
// Blocks that go to one sum in TMEM.  The tensor core cuts off what it adds to a sum
// where an fp32 addition rounds, 2^-23 of it at most for each product of sixteen keys:
// 64 blocks lose 5e-5 of the result where the values have a mean (limit 2^-14), 1024
// blocks in one sum 8.3e-4, more than the output's rounding to fp16.  So every 64 blocks
// a row's sums are put aside, and added to what lies there, in fp32 (1300 tokens at the
// end of 131072, 64 / 1 heads: 5.05 ms, 5.02 in one sum).
constexpr int kPrSum = 64;

// One piece of work: kPrRows query rows of a sequence (a row is a (token, head
// of the group) pair, q = t G + g, so a tile is full whatever G is and spans
// few positions) against key blocks [blk0, blk1), for each key/value head.
struct PromptItem {
  int seq, off, len, pos0;         // sequence, its first packed row, tokens, first position
  int row0, blk0, blk1, split;     // first query row; the split-th of
  int nsplit, rec, group, unused;  // nsplit pieces, which meet through records rec ..
};

struct PromptWork {
  int items;           // of all sequences, heads apart
  int groups;          // tiles whose keys are split
  PromptItem* item;
  unsigned int* done;  // [groups, Hkv, 2] pieces that have arrived
  uint8_t* odd;        // [Hkv, N] a value of this row is not finite
  float* rec;          // partial results: [record, Hkv, 2][kPrRec]
};
// m, l and the weighted values of 128 rows, a row's next value 128 floats on
constexpr int kPrRec = (kHeadDim + 2) * 128;

struct PromptLayout {
  int64_t max_items, max_recs;
  size_t item, done, odd, q, rec, aside, bytes;
};

// Pieces that a launch may split its work into: twice the SMs.
static int64_t prompt_max_pieces() { return 2 * (int64_t)device_sm_count(); }

static PromptLayout prompt_layout(int B, int64_t N, int Hq, int Hkv, int64_t max_ctx) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  PromptLayout l;
  const int64_t tiles = N * (Hq / Hkv) / kPrRows + B;
  const int64_t blocks = (max_ctx + kPrKeys - 1) / kPrKeys;
  const int64_t pieces = prompt_max_pieces();
  l.max_recs = blocks < 3 ? 0 : tiles * blocks * Hkv < pieces ? tiles * blocks * Hkv : pieces;
  l.max_items = tiles > pieces ? tiles : l.max_recs > tiles ? l.max_recs : tiles;
  l.item = up(sizeof(PromptWork));
  l.done = l.item + up((size_t)l.max_items * sizeof(PromptItem));
  l.odd = l.done + up((size_t)l.max_recs * 2 * sizeof(unsigned int));
  l.q = l.odd + up((size_t)Hkv * N);
  l.rec = l.q + up((size_t)N * Hq * kHeadDim * sizeof(__half));
  l.aside = l.rec + up((size_t)l.max_recs * 2 * kPrRec * sizeof(float));
  l.bytes = l.aside + (blocks > kPrSum ? (size_t)device_sm_count() * 2 * kPrRec * sizeof(float) : 0);
  return l;
}

size_t prompt_workspace_bytes(int B, int64_t N, int Hq, int Hkv, int64_t max_ctx) {
  return prompt_layout(B, N, Hq, Hkv, max_ctx).bytes;
}

// ---- the schedule --------------------------------------------------------------

struct PlanArgs {
  Packed pk;
  int G, Hkv, sms;
  int64_t max_pieces;
  PromptWork* work;
  PromptWork init;
};

// The batch's offsets and positions, in shared memory where they fit (the plan
// walks them five times, and every walk would wait for memory).
constexpr int kPlanSeqs = 512;
struct PlanBatch {
  int off[kPlanSeqs + 1], pos[kPlanSeqs];
};

// Calls f(b, off, len, p0, row0, blocks) for every tile of every sequence that
// fits its cache; a warp a sequence, a lane a tile.
template <typename F>
__device__ __forceinline__ void for_tiles(const PlanArgs& a, const PlanBatch& s, F f) {
  const int lane = threadIdx.x & 31;
  const bool near = a.pk.B <= kPlanSeqs;
  for (int b = threadIdx.x >> 5; b < a.pk.B; b += blockDim.x >> 5) {
    const int off = near ? s.off[b] : a.pk.offsets[b], len = (near ? s.off[b + 1] : a.pk.offsets[b + 1]) - off;
    const int64_t p0 = near ? s.pos[b] : a.pk.pos0[b];
    if (p0 < 0 || p0 + len > a.pk.max_ctx) continue;
    const int64_t rows = (int64_t)len * a.G;
    for (int64_t r = (int64_t)lane * kPrRows; r < rows; r += 32 * kPrRows) {
      const int64_t last = min(r + kPrRows, rows) - 1;
      const int blocks = (int)((p0 + last / a.G) / kPrKeys) + 1;
      f(b, off, len, (int)p0, (int)r, blocks);
    }
  }
}

// Tiles in order of falling cost, so that the persistent CTAs, who take items in
// turn, end together.  Few tiles (a short chunk behind a long prefix) are cut
// along the keys: of pieces of half to twice an SM's even share of the blocks, or
// no cut, the cheapest by rounds over the SMs x (blocks of the longest piece + 3
// for what a piece costs besides).  This CTA runs beside the ones that rotate, and
// for short prompts it is the longest: few tiles are listed in shared memory and
// ordered by counting, in three steps.
constexpr int kPlanCuts = 13, kPlanTiles = 320;
__device__ void prompt_plan(const PlanArgs& a) {
  __shared__ unsigned int start[kPrMaxBlocks + 1];
  __shared__ unsigned int tiles, longest, total, items, groups, recs, warp_sum_[8], cost[kPlanCuts];
  __shared__ int tile_seq[kPlanTiles], tile_row[kPlanTiles], tile_blocks[kPlanTiles];
  __shared__ PlanBatch batch;
  const int tid = threadIdx.x, lane = tid & 31;
  bool bad = false;
  for (int b = tid; b < a.pk.B; b += blockDim.x) {
    const int lo = a.pk.offsets[b], hi = a.pk.offsets[b + 1];
    bad |= lo < 0 || hi < lo || (int64_t)hi > a.pk.N;
    if (b < kPlanSeqs) {
      batch.off[b] = lo;
      batch.off[b + 1] = hi;  // (the next sequence's thread writes the same)
      batch.pos[b] = a.pk.pos0[b];
    }
  }
  if (tid == 0) tiles = longest = total = items = groups = recs = 0;
  for (int i = tid; i <= kPrMaxBlocks; i += blockDim.x) start[i] = 0;
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      atomicOr(&g_prompt_status, SQ_DEV_BAD_POSITION);
      *a.work = a.init;
    }
    return;
  }
  for_tiles(a, batch, [&](int b, int, int, int, int row0, int blocks) {
    const unsigned int i = atomicAdd(&tiles, 1u);
    if (i < kPlanTiles) {
      tile_seq[i] = b;
      tile_row[i] = row0;
      tile_blocks[i] = blocks;
      atomicAdd(&total, (unsigned)blocks);  // (needed of a listed batch only)
      atomicMax(&longest, (unsigned)blocks);
    }
  });
  __syncthreads();
  auto emit = [&](int b, int row0, int blocks, unsigned int S, unsigned int at) {
    const int off = a.pk.B <= kPlanSeqs ? batch.off[b] : a.pk.offsets[b];
    const int end = a.pk.B <= kPlanSeqs ? batch.off[b + 1] : a.pk.offsets[b + 1];
    const int p0 = a.pk.B <= kPlanSeqs ? batch.pos[b] : a.pk.pos0[b];
    PromptItem it = {b, off, end - off, p0, row0, 0, 0, 0, (int)S, -1, -1, 0};
    if (S > 1) {
      it.group = (int)atomicAdd(&groups, 1u);
      it.rec = (int)atomicAdd(&recs, S);
      for (int i = 0; i < 2 * a.Hkv; ++i) a.init.done[(int64_t)it.group * 2 * a.Hkv + i] = 0;
    }
    for (unsigned int s = 0; s < S; ++s) {
      it.split = (int)s;
      it.blk0 = (int)((unsigned)blocks * s / S);
      it.blk1 = (int)((unsigned)blocks * (s + 1) / S);
      a.init.item[at + s] = it;
    }
  };
  if (tiles <= kPlanTiles) {
    const int n = (int)tiles;
    unsigned int chunk = kPrMaxBlocks + 1;
    if ((int64_t)n * a.Hkv < a.max_pieces && longest > 2) {
      const unsigned int even = (total * a.Hkv + (unsigned)a.sms - 1) / (unsigned)a.sms;
      auto cut = [&](int i) { return max(2u, (even * (4 + i) + 7) / 8); };
      for (int i = tid >> 5; i < kPlanCuts; i += (int)(blockDim.x >> 5)) {
        const unsigned int c = cut(i);
        unsigned int pieces = 0, piece = 0;
        for (int t = lane; t < n; t += 32) {
          const unsigned int x = (unsigned)tile_blocks[t], S = (x + c - 1) / c;
          pieces += S;
          piece = max(piece, (x + S - 1) / S);
        }
        pieces = __reduce_add_sync(0xffffffffu, pieces) * a.Hkv;
        piece = __reduce_max_sync(0xffffffffu, piece);
        if (lane == 0)
          cost[i] = (int64_t)pieces > a.max_pieces ? 0xffffffffu
                                                   : (pieces + a.sms - 1) / (unsigned)a.sms * (piece + 3);
      }
      __syncthreads();
      // uncut: the longest tile, or the tiles in rounds of their mean
      unsigned int best = longest + 2;
      const unsigned int rounds = ((unsigned)n * a.Hkv + a.sms - 1) / (unsigned)a.sms;
      if (rounds > 1) best = max(best, rounds * (total / (unsigned)n + 2));
      for (int i = 0; i < kPlanCuts; ++i)
        if (cost[i] < best) {
          best = cost[i];
          chunk = cut(i);
        }
    }
    for (int t = tid; t < n; t += blockDim.x) {
      const unsigned int x = (unsigned)tile_blocks[t], S = (x + chunk - 1) / chunk, piece = (x + S - 1) / S;
      unsigned int at = 0;  // pieces of the tiles before it
      for (int u = 0; u < n; ++u) {
        const unsigned int y = (unsigned)tile_blocks[u], Su = (y + chunk - 1) / chunk, pu = (y + Su - 1) / Su;
        if (pu > piece || (pu == piece && u < t)) at += Su;
      }
      emit(tile_seq[t], tile_row[t], (int)x, S, at);
      atomicAdd(&items, S);
    }
  } else {
    // many: a counting sort by their blocks, uncut
    for_tiles(a, batch, [&](int, int, int, int, int, int blocks) { atomicAdd(&start[blocks], 1u); });
    __syncthreads();
    // positions: the largest bin first
    constexpr int kPer = (kPrMaxBlocks + kPrPrepThreads) / kPrPrepThreads;
    unsigned int v[kPer], sum = 0;
    const int hi = kPrMaxBlocks - tid * kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = hi - i >= 0 ? start[hi - i] : 0;
      sum += v[i];
    }
    unsigned int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned int n = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += n;
    }
    if (lane == 31) warp_sum_[tid >> 5] = run;
    __syncthreads();
    run -= sum;
    for (int w = 0; w < (tid >> 5); ++w) run += warp_sum_[w];
    if (tid == kPrPrepThreads - 1) items = run + sum;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (hi - i >= 0) start[hi - i] = run;
      run += v[i];
    }
    __syncthreads();
    for_tiles(a, batch, [&](int b, int, int, int, int row0, int blocks) {
      emit(b, row0, blocks, 1u, atomicAdd(&start[blocks], 1u));
    });
  }
  __syncthreads();
  if (tid == 0) {
    PromptWork w = a.init;
    w.items = (int)items;
    w.groups = (int)groups;
    *a.work = w;
  }
}

// ---- rotation and append -------------------------------------------------------

__device__ __forceinline__ bool any_nonfinite8(uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7c00u) == 0x7c00u || (w[i] & 0x7c000000u) == 0x7c000000u;
  return odd;
}

// CTA 0 plans; the others take R rows each: the rotated queries into
// the workspace, [Hkv, N, G, D], the rotated keys and the values into the
// caches.  A sequence that does not fit its cache writes nothing there, and
// zeros to its rows of `out`.  16 bytes (eight values) a thread and access, of
// both halves of a head for the rotation; bound by these bytes for long
// prompts (the queries are written once and read once more than they must: 8000
// rows of 40 / 8 heads 50 us, 4.6 TB/s).  Rows of a CTA share the look at the
// offsets; with few of them a CTA's chain counts, with many the CTAs (call of 300
// rows R = 1, 2, 4: 90, 92, 99 us, of 2900 47.8, 47.1, 48.8, of 8000 550, 544, 544).
constexpr int64_t kPrFewRows = 1024;  // up to here R = 1, above 2
template <int R>
__global__ void __launch_bounds__(kPrPrepThreads) prompt_prepare_kernel(
    const __half* __restrict__ qkv, int Hq, const RopeFreq rf, const __grid_constant__ PlanArgs a,
    __half* __restrict__ kc, __half* __restrict__ vc, __half* __restrict__ qr, __half* __restrict__ out) {
  griddep_wait();
  griddep_launch_dependents();
  if (blockIdx.x == 0) {
    prompt_plan(a);
    return;
  }
  const Packed& pk = a.pk;
  const int G = a.G, Hkv = a.Hkv, tid = threadIdx.x;
  __shared__ RopeCS cs[R][kHeadDim / 2];
  __shared__ float2 csq[R][kHeadDim / 2];  // the heads, for queries
  __shared__ int seq[R], pos[R];
  const int64_t row0 = (int64_t)(blockIdx.x - 1) * R;
  if (packed_rows<R>(pk, row0, seq, pos, &g_prompt_status)) return;
  if (tid < R * (kHeadDim / 2)) {
    const int i = tid / (kHeadDim / 2), d = tid % (kHeadDim / 2);
    // (eight neighbouring dimensions lie 128 bytes apart, so that the lanes of a head read neighbours)
    if (seq[i] >= 0 && pos[i] >= 0) {
      const RopeCS r = rope_cs_pair(pos[i], rf.f[d]);
      cs[i][(d & 7) * 8 + (d >> 3)] = r;
      csq[i][(d & 7) * 8 + (d >> 3)] = make_float2(r.c.h, r.s.h);
    }
  }
  __syncthreads();
  const int64_t width = (int64_t)(Hq + 2 * Hkv) * kHeadDim;
  const int tasks = (Hq + Hkv) * 8;
  for (int idx = tid; idx < R * tasks; idx += kPrPrepThreads) {
    const int i = idx / tasks, r = idx - i * tasks, h = r >> 3, u = r & 7;
    const int64_t row = row0 + i;
    const int b = seq[i];
    if (b < 0) continue;
    if (pos[i] < 0) {
      if (h < Hq) {
        uint4* o = reinterpret_cast<uint4*>(out + row * Hq * kHeadDim + h * kHeadDim + u * 8);
        o[0] = o[8] = make_uint4(0, 0, 0, 0);
      }
      continue;
    }
    const uint4* src = reinterpret_cast<const uint4*>(qkv + row * width + (int64_t)h * kHeadDim + u * 8);
    const uint4 x1 = src[0], x2 = src[8];
    const __half* e1 = reinterpret_cast<const __half*>(&x1);
    const __half* e2 = reinterpret_cast<const __half*>(&x2);
    uint4 y1, y2;
    __half* z1 = reinterpret_cast<__half*>(&y1);
    __half* z2 = reinterpret_cast<__half*>(&y2);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __half2float(e1[e]), q = __half2float(e2[e]);
      // queries: fp32 does (one in 5000 to the other fp16 neighbour).  They are operands of
      // the tensor core, which takes fp16 beside the caches' fp16 keys; a second term for
      // what the rounding leaves would double the scores' products, half of all.  With the
      // weights' rounding the result is off by 2.2e-4 to 2.9e-4, by 1.9e-4 to 2.1e-4 without
      if (h < Hq) {
        const float2 c = csq[i][e * 8 + u];
        z1[e] = __float2half_rn(p * c.x - q * c.y);
        z2[e] = __float2half_rn(q * c.x + p * c.y);
      } else {
        const RopeCS c = cs[i][e * 8 + u];
        z1[e] = rope_f16(p, c.c, -q, c.s);
        z2[e] = rope_f16(q, c.c, p, c.s);
      }
    }
    __half* dst = h < Hq ? qr + (((int64_t)(h / G) * pk.N + row) * G + h % G) * kHeadDim
                         : kc + (((int64_t)b * Hkv + h - Hq) * pk.max_ctx + pos[i]) * kHeadDim;
    reinterpret_cast<uint4*>(dst + u * 8)[0] = y1;
    reinterpret_cast<uint4*>(dst + u * 8)[8] = y2;
  }
  // values: 16 lanes a head's row (whole warps go round together, as they vote: one row
  // of an odd number of heads leaves the last half of one without a part)
  const int parts = R * Hkv * 16;
  for (int idx = tid; idx - (tid & 31) < parts; idx += kPrPrepThreads) {
    const int at = min(idx, parts - 1), i = at / (Hkv * 16), r = at - i * (Hkv * 16), h = r >> 4, u = r & 15;
    const int64_t row = row0 + i;
    const bool mine = idx < parts && seq[i] >= 0 && pos[i] >= 0;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (mine) {
      x = reinterpret_cast<const uint4*>(qkv + row * width + (int64_t)(Hq + Hkv + h) * kHeadDim)[u];
      reinterpret_cast<uint4*>(vc + (((int64_t)seq[i] * Hkv + h) * pk.max_ctx + pos[i]) * kHeadDim)[u] = x;
    }
    const unsigned int odd = __ballot_sync(0xffffffffu, any_nonfinite8(x));
    if (mine && u == 0) a.init.odd[(int64_t)h * pk.N + row] = (odd >> (tid & 16)) & 0xffffu ? 1 : 0;
  }
}

// ---- attention -----------------------------------------------------------------

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2,
                                            uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}

// The A operand from TMEM (probabilities, two fp16 a column).
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                              uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.u32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Descriptor of a value tile, rows of keys (K) with the head dimension (N)
// running: 64 dimensions of a key are one 128-byte swizzle row, eight keys an
// atom of 1024 bytes (stride), the next 64 dimensions 16 KB on (leading).
__device__ __forceinline__ uint64_t sw128_desc_mn(uint32_t saddr) {
  uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((kPrTile / 2) >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

struct PromptArgs {
  const PromptWork* work;
  const __half* vc;
  __half* out;
  float* aside;  // sums put aside: [CTA, 2][kPrRec]
  int Hq, Hkv, G;
  int64_t N, max_ctx;
};

// Scores become weights 2^(s c - m c + kPrBias), c = log2(e) / sqrt(D): up to
// 2^(kPrBias + kPrSlack) they are below fp16's largest value, and those down to
// 2^-24 of the row's maximum keep all of fp16's bits.
constexpr float kPrBias = 10.0f, kPrSlack = 5.0f;

constexpr int kPrThreads = 384;
constexpr int kPrOffKV = 2 * kPrTile;  // behind the queries
constexpr int kPrOffBar = kPrOffKV + (kPrK + kPrV) * kPrTile;
constexpr int kPrSmem = kPrOffBar + 512 + 1024;  // and room to align the tiles to 1024 bytes

struct PromptBars {
  uint64_t q_full, q_empty, k_full[kPrK], k_empty[kPrK], v_full[kPrV], v_empty[kPrV], v_ready[kPrV], s_full[2],
      p_ready[2][2], o_done[2], drain;
  uint32_t tmem;
  int dead;     // a wait has run out: no one waits any more
  int odd[8];   // [round % 8]: 1 + the round in which a value that is not finite was met (the
                // values' warps are at most kPrV blocks ahead)
  int last[2];  // this half's piece was the last of its group to arrive
};
static_assert(sizeof(PromptBars) <= 512, "barriers fit their place");

// Waits at most two seconds, and not at all once another wait has run out.
__device__ __forceinline__ bool pr_wait(uint32_t bar, uint32_t parity, PromptBars* s) {
  return tc_wait(bar, parity, &s->dead, &g_prompt_status);
}
__device__ __forceinline__ void pr_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// The blocks of an item that half h of its rows sees any key of.
__device__ __forceinline__ int pr_blocks(const PromptItem& it, int G, int h) {
  const int rows = it.len * G;
  if (it.row0 + h * 128 >= rows) return 0;
  const int last = min(it.row0 + h * 128 + 128, rows) - 1;
  return max(min(it.blk1, (it.pos0 + last / G) / kPrKeys + 1) - it.blk0, 0);
}

// One persistent CTA an SM, twelve warps: two groups of four softmax warps, one
// for each half (128 rows) of an item's queries, a TMA warp, an MMA warp, and two
// that look after the values.
//
// Per block of 128 keys and half: S = Q K^T (128 x 128 fp32 in TMEM) by
// tcgen05.mma from shared memory; a softmax thread owns a row, reads it, and
// writes its weights as fp16 over it; O += P V takes the weights from TMEM and
// the values from shared memory.  The tensor pipe works on one half while the
// other is in its softmax.  TMEM: S0, S1, O0, O1, 128 columns each.
// The running maximum of a row is let lag by up to 2^kPrSlack before O and the
// sum are rescaled (the result is the same but for fp16's range), so that O
// leaves TMEM once, at the end, and (Long) every kPrSum blocks before it.  Long is
// for caches of more than kPrSum blocks: its code, though not run, made a call of 20
// tokens take 12.5 us instead of 11.9.
// Bound: the chain of a half's block (scores, softmax, weights, products), as its
// scores have one place.  8000 tokens, 40 / 8 heads: 485 us, 1.35 PFLOP/s, the
// tensor pipe busy for 59 % of them; 1.83 us for both halves' block, 1.06 of them
// products.  Scores of 64 keys in two places (the next ones are there before the
// weights are) cost 735 us for the call instead of 541: twice the hand-overs, and
// products of 64 columns; sixteen softmax warps 554; exponentials of the first 64
// keys before the block's maximum is known 547.
template <bool Long>
__global__ void __launch_bounds__(kPrThreads, 1)
    prompt_attention_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                            const __grid_constant__ CUtensorMap tv, const PromptArgs a) {
  extern __shared__ uint8_t pr_raw[];
  uint8_t* smem = pr_raw + (((smem_u32(pr_raw) + 1023u) & ~1023u) - smem_u32(pr_raw));
  PromptBars* s = reinterpret_cast<PromptBars*>(smem + kPrOffBar);
  const uint32_t base = smem_u32(smem);
#define PR_BAR(member) (bars + (uint32_t)offsetof(PromptBars, member))
  const uint32_t bars = base + kPrOffBar;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(&s->q_full, 1);
    mbar_init(&s->q_empty, 1);
    for (int i = 0; i < kPrK; ++i) {
      mbar_init(&s->k_full[i], 1);
      mbar_init(&s->k_empty[i], 1);
    }
    for (int i = 0; i < kPrV; ++i) {
      mbar_init(&s->v_full[i], 1);
      mbar_init(&s->v_empty[i], 1);
      mbar_init(&s->v_ready[i], 2);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(&s->s_full[h], 1);
      mbar_init(&s->p_ready[h][0], 4);
      mbar_init(&s->p_ready[h][1], 4);
      mbar_init(&s->o_done[h], 1);
    }
    mbar_init(&s->drain, 1);
    s->dead = 0;
    for (int i = 0; i < 8; ++i) s->odd[i] = 0;
    fence_mbar_init();
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s->tmem)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&s->tmem;
  griddep_wait();
  griddep_launch_dependents();
  const PromptItem* items = a.work->item;
  const int total = a.work->items * a.Hkv;  // (below 2^31: rows * Hq <= 2^30)
  // round r of this CTA: forwards and backwards in turn, as costs fall along the list
  auto pick = [&](int r) {
    return r * (int)gridDim.x + ((r & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
  };

  // registers: 384 threads x 168 at launch; the softmax groups take 208, the
  // others keep 88 (256 x 208 + 128 x 88 = 384 x 168); with 72 those spilled in
  // their loops (with 88 the kernel still spills 64 bytes, Long 84)
  if (warp >= 8) {
   asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
   if (warp == 8) {
    if (lane == 0) {
      // ------------------------------------------------------------- TMA
      // Every waiter of a barrier waits for each of its phases, so that a parity
      // names one phase: keys and values have rings of their own.
      uint32_t nk = 0, nv = 0;  // tiles requested
      bool fine = true;
      auto tile = [&](const CUtensorMap* map, uint32_t full, uint32_t empty, uint32_t dst, uint32_t lap, int blk,
                      int bh) {
        if (!(fine = pr_wait(empty, (lap & 1u) ^ 1u, s))) return;
        pr_expect(full, kPrTile);
        tma_load_3d(dst, map, 0, blk * kPrKeys, bh, full);
        tma_load_3d(dst + kPrTile / 2, map, 64, blk * kPrKeys, bh, full);
      };
      int done = 0;  // items whose queries were requested
      for (int r = 0, w; fine && (w = pick(r)) < total; ++r) {
        const PromptItem it = items[w / a.Hkv];
        const int kvh = w % a.Hkv, bh = it.seq * a.Hkv + kvh;
        const int nb = max(pr_blocks(it, a.G, 0), pr_blocks(it, a.G, 1));
        const bool two = it.row0 + 128 < it.len * a.G;
        for (int j = 0; fine && j < nb; ++j) {
          tile(&tk, PR_BAR(k_full) + 8 * (nk % kPrK), PR_BAR(k_empty) + 8 * (nk % kPrK), base + kPrOffKV + (nk % kPrK) * kPrTile, nk / kPrK,
               it.blk0 + j, bh);
          if (!fine) break;
          ++nk;
          if (j == 0) {
            if (!(fine = pr_wait(PR_BAR(q_empty), ((uint32_t)r & 1u) ^ 1u, s))) break;
            const int64_t y = ((int64_t)kvh * a.N + it.off) * a.G + it.row0;
            pr_expect(PR_BAR(q_full), two ? 2 * kPrTile : kPrTile);
            for (int h = 0; h < (two ? 2 : 1); ++h)
              for (int c = 0; c < 2; ++c)
                tma_load_q(base + h * kPrTile + c * (kPrTile / 2), &tq, 64 * c, (int)(y + 128 * h), PR_BAR(q_full));
            ++done;
          }
          tile(&tv, PR_BAR(v_full) + 8 * (nv % kPrV), PR_BAR(v_empty) + 8 * (nv % kPrV), base + kPrOffKV + (kPrK + nv % kPrV) * kPrTile,
               nv / kPrV, it.blk0 + j, bh);
          if (fine) ++nv;
        }
      }
      if (!fine) {  // no copy may land after the CTA has left
        for (uint32_t i = nk > kPrK ? nk - kPrK : 0; i < nk; ++i)
          mbar_wait_bounded(&s->k_full[i % kPrK], (i / kPrK) & 1u, 1u << 20);
        for (uint32_t i = nv > kPrV ? nv - kPrV : 0; i < nv; ++i)
          mbar_wait_bounded(&s->v_full[i % kPrV], (i / kPrV) & 1u, 1u << 20);
        if (done) mbar_wait_bounded(&s->q_full, (uint32_t)(done - 1) & 1u, 1u << 20);
      }
    }
   } else if (warp == 9) {
    if (lane == 0) {
      // ------------------------------------------------------------- MMA
      // D fp32, A and B fp16, M = N = 128; of the values N runs (bit 16)
      const uint32_t id_qk = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
      const uint32_t id_pv = id_qk | (1u << 16);
      uint32_t nk = 0, nv = 0;  // tiles of keys, of values taken
      uint32_t np[2] = {0, 0};  // blocks of each half whose weights were waited for
      bool fine = true;
      auto qk = [&](int h, uint32_t st) {
        const uint64_t qd = sw128_desc(base + h * kPrTile), kd = sw128_desc(base + kPrOffKV + st * kPrTile);
#pragma unroll
        for (int kk = 0; kk < kHeadDim / 16; ++kk) {
          const uint64_t o = (uint64_t)((kk >> 2) * (kPrTile / 2 / 16) + (kk & 3) * 2);
          tc_mma_f16(tmem + h * 128, qd + o, kd + o, id_qk, kk > 0);
        }
        tc_commit_at(PR_BAR(s_full) + 8 * (h));
      };
      for (int r = 0, w; fine && (w = pick(r)) < total; ++r) {
        const PromptItem it = items[w / a.Hkv];
        const int nb[2] = {pr_blocks(it, a.G, 0), pr_blocks(it, a.G, 1)};
        const int nm = max(nb[0], nb[1]);  // (never zero: the item's last row sees its last block)
        auto keys = [&]() { return pr_wait(PR_BAR(k_full) + 8 * (nk % kPrK), (nk / kPrK) & 1u, s); };
        if (!(fine = keys() && pr_wait(PR_BAR(q_full), (uint32_t)r & 1u, s))) break;
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (nb[h] > 0) qk(h, nk % kPrK);
        tc_commit_at(PR_BAR(k_empty) + 8 * (nk % kPrK));
        ++nk;
        if (nm == 1) tc_commit_at(PR_BAR(q_empty));
        for (int j = 0; fine && j < nm; ++j) {
          if (j + 1 < nm && !(fine = keys())) break;
          if (!(fine = pr_wait(PR_BAR(v_ready) + 8 * (nv % kPrV), (nv / kPrV) & 1u, s))) break;
          const uint64_t vd = sw128_desc_mn(base + kPrOffKV + (kPrK + nv % kPrV) * kPrTile);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (j >= nb[h]) continue;
            // the first 64 keys' weights are there while the others are computed
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              if (!(fine = pr_wait(PR_BAR(p_ready) + 16 * (h) + 8 * (half), np[h] & 1u, s))) break;
              tc_fence_after();
#pragma unroll
              for (int kk = 4 * half; kk < 4 * half + 4; ++kk)
                tc_mma_f16_ts(tmem + 256 + h * 128, tmem + h * 128 + kk * 8, vd + kk * (16 * 128 / 16), id_pv,
                              (Long ? j % kPrSum : j) > 0 || kk > 0);
            }
            if (!fine) break;
            ++np[h];
            tc_commit_at(PR_BAR(o_done) + 8 * (h));
            if (j + 1 < nb[h]) qk(h, nk % kPrK);
          }
          if (!fine) break;
          tc_commit_at(PR_BAR(v_empty) + 8 * (nv % kPrV));
          ++nv;
          if (j + 1 < nm) {
            tc_commit_at(PR_BAR(k_empty) + 8 * (nk % kPrK));
            ++nk;
          }
          if (j + 2 == nm) tc_commit_at(PR_BAR(q_empty));
        }
      }
      if (!fine) {  // what was issued still writes TMEM
        tc_commit_at(PR_BAR(drain));
        mbar_wait_bounded(&s->drain, 0u, 1u << 20);
      }
    }
   } else {
    // ------------------------------------------------------------- values
    // A weight of zero must not meet a value that is not finite: cache rows
    // behind the sequence's last token become zero in the tile, and so do such
    // values of new tokens (their rows are marked), which go to the rows that
    // see them at the end, by themselves.
    const int t = tid - 320;
    uint32_t nv = 0;
    bool fine = true;
    for (int r = 0, w; fine && (w = pick(r)) < total; ++r) {
      const PromptItem it = items[w / a.Hkv];
      const uint8_t* odd = a.work->odd + (int64_t)(w % a.Hkv) * a.N + it.off;
      const int nb = max(pr_blocks(it, a.G, 0), pr_blocks(it, a.G, 1)), end = it.pos0 + it.len;
      // the marks of a block are read a block ahead: what a tile waits for here is
      // in the chain of every tile (with the read in it, and a fence that nothing
      // needed, the call of 8000 tokens took 14 us more)
      auto marks = [&](int j) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = (it.blk0 + j) * kPrKeys + t + 64 * e;
          if (j < nb && key >= it.pos0 && key < end && odd[key - it.pos0]) m |= 1u << e;
        }
        return m;
      };
      uint32_t next = marks(0);
      for (int j = 0; j < nb; ++j, ++nv) {
        const uint32_t st = nv % kPrV, ph = (nv / kPrV) & 1u;
        const int key0 = (it.blk0 + j) * kPrKeys;
        const uint32_t marked = next;
        next = marks(j + 1);
        fine = __all_sync(0xffffffffu, pr_wait(PR_BAR(v_full) + 8 * (st), ph, s));
        if (!fine) break;
        const int gone = min(max(key0 + kPrKeys - end, 0), kPrKeys);
        if (__any_sync(0xffffffffu, gone > 0 || marked)) {
          uint8_t* v = smem + kPrOffKV + (kPrK + st) * kPrTile;
          for (int i = t; i < gone * 16; i += 64)
            *reinterpret_cast<uint4*>(v + ((i >> 3) & 1) * (kPrTile / 2) + (kPrKeys - gone + (i >> 4)) * 128 +
                                      (i & 7) * 16) = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if ((marked >> e) & 1) {
              for (int c = 0; c < 2; ++c)
                for (int d = 0; d < 64; ++d) {
                  uint16_t* x = reinterpret_cast<uint16_t*>(v + c * (kPrTile / 2) + (t + 64 * e) * 128) + d;
                  if ((*x & 0x7c00u) == 0x7c00u) *x = 0;
                }
              *(volatile int*)&s->odd[r & 7] = r + 1;
            }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        if (lane == 0) tc_arrive(PR_BAR(v_ready) + 8 * (st));
      }
    }
   }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ------------------------------------------------------------- softmax
    const int h = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + h * 128 + lanes, to = tmem + 256 + h * 128 + lanes;
    const float c = 0.08838834764831845f * 1.4426950408889634f;
    uint32_t ns = 0;  // blocks of this half
    for (int r = 0, w; (w = pick(r)) < total; ++r) {
      const PromptItem it = items[w / a.Hkv];
      const int kvh = w % a.Hkv;
      if (it.row0 + h * 128 >= it.len * a.G) continue;
      const int nb = pr_blocks(it, a.G, h);
      const int q = it.row0 + h * 128 + row;
      const bool mine = q < it.len * a.G;
      const int tok = (mine ? q : it.len * a.G - 1) / a.G, pos = it.pos0 + tok;
      const int first = __shfl_sync(0xffffffffu, pos, 0);  // the warp's first position
      float m = -INFINITY;
      unsigned long long l2 = 0;  // the sum, two halves
      for (int j = 0; j < nb; ++j, ++ns) {
        pr_wait(PR_BAR(s_full) + 8 * (h), ns & 1u, s);
        if (j > 0) pr_wait(PR_BAR(o_done) + 8 * (h), (ns & 1u) ^ 1u, s);
        __syncwarp();
        tc_fence_after();
        if (Long && j % kPrSum == 0 && j > 0) {  // (this block's products begin a sum, once its weights are there)
          float* aside = a.aside + (int)(blockIdx.x * 2 + h) * kPrRec + row;
          const float2 lp = f2unpack(l2);
          float f = 0.0f, la = lp.x + lp.y;
          l2 = 0;
          if (j > kPrSum) {
            const float ma = __ldcg(aside + kHeadDim * 128);
            if (ma != -INFINITY) f = ex2((ma - m) * c);
            la = fmaf(__ldcg(aside + (kHeadDim + 1) * 128), f, la);
          }
          __stcg(aside + kHeadDim * 128, m);
          __stcg(aside + (kHeadDim + 1) * 128, la);
#pragma unroll 1
          for (int i = 0; i < kHeadDim; i += 16) {
            uint32_t o[16];
            tm_ld16(to + i, o);
            tm_wait_ld();
            tm_loaded16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x = __uint_as_float(o[e]);
              if (j > kPrSum) x = fmaf(f, __ldcg(aside + (i + e) * 128), x);
              __stcg(aside + (i + e) * 128, x);
            }
          }
        }
        // scores in two loads, the second under the first one's maximum
        uint32_t v[128];
        const int key0 = (it.blk0 + j) * kPrKeys;
        const bool edge = key0 + kPrKeys - 1 > first;
        const int seen = pos - key0;  // the last key this row sees
        float mx[4];
        tm_ld32(ts, v);
        tm_ld32(ts + 32, v + 32);
        tm_wait_ld();
        tm_loaded32(v);
        tm_loaded32(v + 32);
        tm_ld32(ts + 64, v + 64);
        tm_ld32(ts + 96, v + 96);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (i) {
            tm_wait_ld();
            tm_loaded32(v + 64);
            tm_loaded32(v + 96);
          }
          if (edge) {
#pragma unroll
            for (int e = 64 * i; e < 64 * i + 64; ++e)
              if (e > seen) v[e] = 0xff800000u;
          }
#pragma unroll
          for (int e = 64 * i; e < 64 * i + 64; e += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float x = __uint_as_float(v[e + k]), y = __uint_as_float(v[e + 4 + k]);
              mx[k] = e == 0 ? fmaxf(x, y) : fmaxf(fmaxf(mx[k], x), y);
            }
        }
        const float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        if (__any_sync(0xffffffffu, (mb - m) * c > kPrSlack)) {
          const float mn = fmaxf(m, mb);
          const float f = m == -INFINITY ? 0.0f : ex2((m - mn) * c);
          m = mn;
          if (Long ? j % kPrSum > 0 : j > 0) {
            const unsigned long long f2 = f2pack(f, f);
            asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(l2) : "l"(f2));
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
              uint32_t o[32];
              tm_ld32(to + 32 * i, o);
              tm_wait_ld();
              tm_loaded32(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tm_st32(to + 32 * i, o);
            }
          }
        }
        const float b0 = m == -INFINITY ? 0.0f : fmaf(-m, c, kPrBias);
        const unsigned long long cc = f2pack(c, c), bb = f2pack(b0, b0);
        unsigned long long sum[2] = {l2, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t p[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float2 x = f2unpack(ffma2_to(
                f2pack(__uint_as_float(v[64 * i + 2 * e]), __uint_as_float(v[64 * i + 2 * e + 1])), cc, bb));
            const float p0 = ex2(x.x), p1 = ex2(x.y);
            sum[e & 1] = fadd2(sum[e & 1], f2pack(p0, p1));
            p[e] = pack_f16x2(p0, p1);
          }
          tm_st32(ts + 32 * i, p);
          tm_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) tc_arrive(PR_BAR(p_ready) + 16 * (h) + 8 * (i));  // (32 arrivals of a warp take turns)
        }
        l2 = fadd2(sum[0], sum[1]);
      }
      // ---- the rows' results
      if (nb > 0) pr_wait(PR_BAR(o_done) + 8 * (h), (ns & 1u) ^ 1u, s);
      __syncwarp();
      tc_fence_after();
      const float2 lp = f2unpack(l2);
      float l = lp.x + lp.y, fa = 0.0f;
      if (Long && nb > kPrSum) {
        const float* aside = a.aside + (int)(blockIdx.x * 2 + h) * kPrRec + row;
        const float ma = __ldcg(aside + kHeadDim * 128);
        if (ma != -INFINITY) fa = ex2((ma - m) * c);
        l = fmaf(__ldcg(aside + (kHeadDim + 1) * 128), fa, l);
#pragma unroll 1
        for (int i = 0; i < kHeadDim; i += 16) {
          uint32_t o[16];
          tm_ld16(to + i, o);
          tm_wait_ld();
          tm_loaded16(o);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            o[e] = __float_as_uint(fmaf(fa, __ldcg(aside + (i + e) * 128), __uint_as_float(o[e])));
          tm_st16(to + i, o);
        }
        tm_wait_st();
      }
      const bool split = it.nsplit > 1;
      const float f = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
      const bool odd = *(volatile int*)&s->odd[r & 7] == r + 1;
      float* rec = a.work->rec + ((((int64_t)it.rec + it.split) * a.Hkv + kvh) * 2 + h) * kPrRec + row;
      __half* out = a.out + ((int64_t)(it.off + tok) * a.Hq + kvh * a.G + (q - tok * a.G)) * kHeadDim;
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        uint32_t o[32];
        if (nb > 0) {
          tm_ld32(to + 32 * i, o);
          tm_wait_ld();
          tm_loaded32(o);
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = nb > 0 ? __float_as_uint(__uint_as_float(o[e]) * f) : 0u;
        if (odd) {
          const uint8_t* od = a.work->odd + (int64_t)kvh * a.N + it.off;
          const int k1 = min(pos, it.blk1 * kPrKeys - 1);
          for (int key = max(it.blk0 * kPrKeys, it.pos0); key <= k1; ++key) {
            if (!od[key - it.pos0]) continue;
            const __half* x = a.vc + (((int64_t)it.seq * a.Hkv + kvh) * a.max_ctx + key) * kHeadDim + 32 * i;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float y = __half2float(x[e]);
              if (!isfinite(y)) o[e] = __float_as_uint(__uint_as_float(o[e]) + y);
            }
          }
        }
        if (split) {
#pragma unroll
          for (int e = 0; e < 32; ++e) __stcg(rec + (32 * i + e) * 128, __uint_as_float(o[e]));
        } else if (mine) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint4 y;
            y.x = pack_f16x2(__uint_as_float(o[8 * e]), __uint_as_float(o[8 * e + 1]));
            y.y = pack_f16x2(__uint_as_float(o[8 * e + 2]), __uint_as_float(o[8 * e + 3]));
            y.z = pack_f16x2(__uint_as_float(o[8 * e + 4]), __uint_as_float(o[8 * e + 5]));
            y.w = pack_f16x2(__uint_as_float(o[8 * e + 6]), __uint_as_float(o[8 * e + 7]));
            reinterpret_cast<uint4*>(out)[4 * i + e] = y;
          }
        }
      }
      tc_fence_before();  // (the next item's products overwrite O)
      if (split) {
        __stcg(rec + kHeadDim * 128, m * c);
        __stcg(rec + (kHeadDim + 1) * 128, l);
        __threadfence();
        named_bar_sync(1 + h, 128);
        if (row == 0) {
          const unsigned int n = atomicAdd(&a.work->done[((int64_t)it.group * a.Hkv + kvh) * 2 + h], 1u);
          s->last[h] = n == (unsigned)it.nsplit - 1;
          __threadfence();
        }
        named_bar_sync(1 + h, 128);
        if (*(volatile int*)&s->last[h]) {
          // the pieces in their order along the keys
          const float* p = a.work->rec + (((int64_t)it.rec * a.Hkv + kvh) * 2 + h) * kPrRec + row;
          const int64_t step = (int64_t)a.Hkv * 2 * kPrRec;
          float M = -INFINITY, L = 0.0f;
          for (int i = 0; i < it.nsplit; ++i) M = fmaxf(M, __ldcg(p + i * step + kHeadDim * 128));
          for (int i = 0; i < it.nsplit; ++i) {
            const float mi = __ldcg(p + i * step + kHeadDim * 128);
            if (mi != -INFINITY) L = fmaf(ex2(mi - M), __ldcg(p + i * step + (kHeadDim + 1) * 128), L);
          }
          const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll 1
          for (int d = 0; d < kHeadDim; d += 16) {
            float o[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = 0.0f;
            for (int i = 0; i < it.nsplit; ++i) {
              const float mi = __ldcg(p + i * step + kHeadDim * 128);
              if (mi == -INFINITY) continue;
              const float wgt = ex2(mi - M);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = fmaf(wgt, __ldcg(p + i * step + (d + e) * 128), o[e]);
            }
            if (mine) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                uint4 y;
                y.x = pack_f16x2(o[8 * e] * inv, o[8 * e + 1] * inv);
                y.y = pack_f16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv);
                y.z = pack_f16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv);
                y.w = pack_f16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv);
                reinterpret_cast<uint4*>(out)[d / 8 + e] = y;
              }
            }
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 9)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

#undef PR_BAR

// [rows, 128] fp16, or [heads, rows, 128]: boxes of 64 values x 128 rows.
static bool prompt_map(CUtensorMap* m, const void* base, int64_t rows, int64_t heads) {
  auto enc = tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)rows, (cuuint64_t)heads};
  const cuuint64_t strides[2] = {kHeadDim * 2, (cuuint64_t)rows * kHeadDim * 2};
  const cuuint32_t box[3] = {64, 128, 1}, step[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, heads ? 3 : 2, const_cast<void*>(base), dims, strides, box, step,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static cudaError_t prompt_ready() {
  static std::mutex mu;
  static bool ready[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!ready[dev]) {
    for (auto* k : {prompt_attention_kernel<false>, prompt_attention_kernel<true>}) {
      e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kPrSmem);
      if (e != cudaSuccess) return e;
    }
    ready[dev] = true;
  }
  return cudaSuccess;
}

cudaError_t launch_prompt(const __half* qkv, const Packed& pk, int Hq, int Hkv, double theta, __half* kc,
                          __half* vc, __half* out, void* ws, cudaStream_t st) {
  cudaError_t e = prompt_ready();
  if (e != cudaSuccess) return e;
  const PromptLayout l = prompt_layout(pk.B, pk.N, Hq, Hkv, pk.max_ctx);
  uint8_t* w = reinterpret_cast<uint8_t*>(ws);
  __half* qr = reinterpret_cast<__half*>(w + l.q);
  CUtensorMap tq, tk, tv;
  if (!prompt_map(&tq, qr, pk.N * Hq, 0) || !prompt_map(&tk, kc, pk.max_ctx, (int64_t)pk.B * Hkv) ||
      !prompt_map(&tv, vc, pk.max_ctx, (int64_t)pk.B * Hkv))
    return cudaErrorInvalidValue;
  PlanArgs a = {};
  a.pk = pk;
  a.G = Hq / Hkv;
  a.Hkv = Hkv;
  a.sms = device_sm_count();
  a.max_pieces = l.max_recs;
  a.work = reinterpret_cast<PromptWork*>(w);
  a.init.item = reinterpret_cast<PromptItem*>(w + l.item);
  a.init.done = reinterpret_cast<unsigned int*>(w + l.done);
  a.init.odd = w + l.odd;
  a.init.rec = reinterpret_cast<float*>(w + l.rec);
  const int rows = pk.N <= kPrFewRows ? 1 : 2;
  e = launch_pdl(rows == 1 ? prompt_prepare_kernel<1> : prompt_prepare_kernel<2>,
                 dim3((unsigned)((pk.N + rows - 1) / rows + 1)), dim3(kPrPrepThreads), 0, st, qkv, Hq,
                 rope_freq(theta), a, kc, vc, qr, out);
  if (e != cudaSuccess) return e;
  PromptArgs p = {a.work, vc, out, reinterpret_cast<float*>(w + l.aside), Hq, Hkv, a.G, pk.N, pk.max_ctx};
  int64_t grid = (pk.N * a.G / kPrRows + pk.B) * Hkv;
  if (l.max_recs > grid) grid = l.max_recs;
  if (grid > a.sms) grid = a.sms;
  return launch_pdl(pk.max_ctx > kPrSum * kPrKeys ? prompt_attention_kernel<true> : prompt_attention_kernel<false>,
                    dim3((unsigned)grid), dim3(kPrThreads), (size_t)kPrSmem, st, tq, tk, tv, p);
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
