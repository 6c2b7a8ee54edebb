// Decode attention of one new token per sequence over a paged cache (BF16, or INT8 codes with one scale per token and KV head),
// with the attention weight of every cached token summed up on the way (msd_attn_decode_paged).
//
//   S_hj = scale q_h.k_j,  P = softmax(S),  out = P V,  weights_j += sum_h P_hj
//
// Bound: HBM.  A token of a KV head is 2 (D + Dv) bytes (BF16) for 2 G (D + Dv) multiply-adds of its G query heads.  An SM takes in
// 44 bytes a nanosecond, 23 a clock, and the warp-level MMAs of that (8, 16 or 24 head slots, used or not) are a fifth of what the pipe does,
// so nothing here waits for the tensor cores, and what counts is that loads never stop.  Hence no roles and no hand-offs: each warp
// keeps a ring of token tiles of its own in flight (cp.async, a row's page looked up a tile ahead), multiplies a tile against the
// query fragments in its registers, keeps its own references, sums and outputs, and meets the other warps of its CTA only when
// a sequence ends.  32 sequences of 2048 to 8192 tokens, 32 / 8 heads of 128, pages of 16, no weights: BF16 106 us (6.3 TB/s, 0.98 of a plain
// copy), INT8 67 (5.2 TB/s; 60 of them are the loads alone).  The kernels of this library whose tiles go through tensor memory
// (tcgen05, a CTA's warps in roles), same box: BF16 without pages 124, INT8 with q and P decomposed 72; 16 query heads a KV head INT8 87 / 161;
// 8 x 32768 INT8 97 / 96.  With more than 8 slots, or INT8, instructions start to count: 128 / 8 heads BF16 118 us.
//
// Fragments (mma m16n8k16): 16 tokens are the rows and 8 heads the columns, so that up to 8 heads waste nothing.  The scores are a C
// fragment; transposed in registers (movmatrix) it is the column fragment of the product of v^T (rows: 16 values of d) with P.  INT8
// codes go from shared memory to registers as bytes and become FP16 pairs there (exact): 1024 + (x + 128) has the byte as its lowest bits, and
// 1152 is taken off, 5 instructions for 4 values (BF16 pairs, sign and magnitude apart: 8).
//
// Precision: q and k (codes) are multiplied exactly and summed in FP32; the sums' error is what an FP32 product has.  P for the
// product with v is two BF16 values, or one FP16 value with 11 bits for codes; one BF16 value made the result's error 1.4 times that of
// its own rounding to BF16.  Of the two, both are above 0 where P is, or an infinite value times them would be no number.
//
// Split over the length: the tiles of all sequences form one list, cut into equal runs; run i is walked by U = KV heads x head groups
// CTAs side by side, one per unit, so that CTAs that run together read neighbouring rows.  The grid is what is resident at once.
// A sequence inside one run is finished there; only the first and the last of a run can be cut, so a CTA leaves at most two
// partial results, whatever the lengths are, and a second kernel joins those and turns the scores into weights.  With few tiles the runs of a
// unit are a cluster, which joins them and adds the weights itself after a barrier: one launch.
//
// Tried and dropped: the last CTA to leave a partial result of a sequence joins them (registers of the tile loop; 32 x 2048-8192
// tokens 122 -> 124 us at best, one of 1001 10.1 -> 9.0); keys and values asked for one by one as soon as their halves of a stage are free
// (more in flight, 122 -> 127, 2 x 100000-131072 164 -> 172); scores kept in L2 by a cache hint (0.5 us).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "paged.cuh"

namespace msd {

namespace {

constexpr int kJoinThreads = 256;
constexpr int kAtOnceWeights = 4;           // positions of a thread whose scores are under way together
constexpr int kClusterTiles = 4, kClusterCtas = 16;     // one kernel: most tiles of a CTA, most CTAs of a unit
constexpr float kHeld = 8.0f;               // how far (log2) a score may exceed its reference before that moves
constexpr float kPUnits = 128.0f;           // INT8: 2^15 / 2^kHeld
// Sums of P and of P v are kept times kDown, so that the sum over 2^31 tokens of P <= 2^kHeld is less than 1 and no sum of finite values
// overflows.  (A power of two: nothing rounds elsewhere.)
constexpr float kDown = 1.8189894035458565e-12f, kUp = 1.0f / kDown;      // 2^-39

struct PagedAttnParams {
  PagedCache c;
  // strides of the cache between blocks and tokens: rows in units of 16 bytes, scales in words (offsets fit 32 bits)
  uint32_t k_block, k_token, v_block, v_token, ks_block, ks_token, vs_block, vs_token;
  const uint16_t* q;
  int64_t q_ld;
  const int32_t* table;
  const int32_t* seqlens;
  int64_t cap;                // most tokens of a sequence that the table (and weights) have room for
  int max_blocks, B, Hq, G, groups, U, runs;
  float scale2;               // softmax scale x log2(e)
  uint16_t* out;
  float* lse;
  float* weights;
  int64_t ld, score_ld;
  int score_heads;            // heads of a position's scores: G, made even
  int slots;                  // head slots of a CTA, 8, 16 or 24
  // workspace
  float* part;                // [CTA][2][rows][Dv]: unnormalised outputs, times kDown
  float* part_ml;             // [CTA][2][rows][2]: maximum (log2), and sum times kDown
  int4* tail;                 // [CTA] {sequence cut at the end of its run or -1, first and last run of that sequence}
  int2* seq_runs;             // [B] {first, last run}
  float* lse2;                // [B, Hq] log2-sum of uncut sequences' scores
  float* scores;              // [B, Hkv, score_ld, score_heads] log2 scores
  int part_rows;              // rows of a partial result: min(G, slots)
  int join_weight_ctas;       // CTAs of the join per (sequence, KV head)
  bool leave_l2;              // keys and values leave L2 first
  unsigned* status;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there, uint64_t policy) {      // zeros where there is nothing
  asm volatile("cp.async.cg.shared.global.L2::cache_hint.L2::128B [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp16_all(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
template <bool kHalfs, bool kFirst = false>      // FP16 or BF16 operands; kFirst: c = a b instead of c += a b
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], const uint2& b) {
  const float z0 = kFirst ? 0.0f : c[0], z1 = kFirst ? 0.0f : c[1], z2 = kFirst ? 0.0f : c[2], z3 = kFirst ? 0.0f : c[3];
  if constexpr (kHalfs)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {      // BF16 values, cut off
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {       // of an 8 x 8 matrix of 16-bit values over the warp
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// bytes kLo and kHi of u, each a code plus 128, as an FP16 pair of the codes: 1024 + u has the byte as its lowest bits
template <int kLo, int kHi>
__device__ __forceinline__ uint32_t codes_f16(uint32_t u) {
  const uint32_t t = __byte_perm(u, 0x64646464u, 0x4040 | kLo | (kHi << 8));
  const uint32_t off = 0x64806480u;                                // 1152
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&t), *reinterpret_cast<const __half2*>(&off));
  return *reinterpret_cast<const uint32_t*>(&d);
}

// DP: D and Dv rounded up to 64, 96, 128, 192 or 256; kHeads: head slots of a CTA, 8, 16 or 24.  A tile of a warp is 16 or 32 tokens, 4 to 16 KB
// of keys and values; the rings of an SM's CTAs hold 144 to 192 KB (BF16), and 130 to 198 KB (INT8), less where registers allow two or three CTAs of small
// tiles: INT8 rows of 64 102 KB with 16 slots and 68 with 24, of 96 100 with 24.  Two stages and as many warps as their registers allow (heads of 128, 32 x
// 2048-8192 tokens: INT8 81 / 85 us, 16 / 16 heads of 80 52 / 57 with more stages and fewer warps; at the same number of warps a third
// stage, 24 x 1024-4096: 16 / 16 heads of 64 INT8 39.9 / 44.0, of 256 99 / 101), but for BF16 with two CTAs an SM (128 / 8 heads of 128: 53.5 with two
// stages, 52.6 with three).  Sizes of 96 and 192 beside the powers of two: 128 / 8 heads of 80 BF16 48 -> 42 us, INT8 45 -> 39, 16 / 16 heads
// of 96 INT8 57 -> 50, of 192 BF16 128 -> 122, INT8 92 -> 78.
template <bool kInt8, int DP, int kHeads>
struct Shape {
  static constexpr int kWarps = !kInt8 && DP == 256 ? 6 : 4;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kEs = kInt8 ? 1 : 2;
  static constexpr int kTok = DP == 64 || (kInt8 && DP <= (kHeads == 8 ? 128 : 192)) ? 32 : 16;
  static constexpr int kRow = DP * kEs;                         // bytes of a row in shared memory
  static constexpr int kHalf = kTok * kRow;                     // keys, then values
  static constexpr int kScale = kInt8 ? kTok * 4 : 0;           // then the scales of both
  static constexpr int kStage = 2 * kHalf + 2 * kScale;
  static constexpr int kCtasPerSm = kHeads == 24         ? 2
                                    : !kInt8 && DP == 256 ? 1
                                    : kInt8 && DP == 64  ? (kHeads == 8 ? 4 : 3)
                                    : DP == 96 || (kHeads == 8 && DP <= (kInt8 ? 192 : 128)) ? 3
                                                         : 2;
  static constexpr bool kQInSmem = (DP == 256 && kHeads == 16) || (DP >= 128 && kHeads == 24);   // (the registers of the outputs leave it no room)
  static constexpr int kQBytes = kQInSmem ? (DP / 16) * (kHeads / 8) * 32 * 8 : 0, kStatic = 2304;
  static constexpr int kStages = !kInt8 && kCtasPerSm == 2 && 2 * kWarps * 3 * kStage <= 200 * 1024 ? 3 : 2;
  static constexpr int kRing = kWarps * kStages * kStage;
  // The warps' outputs meet in the stages that their last tiles left, all heads or 8 at a time; rows four words apart in the banks
  // where there is room for that.
  static constexpr int kMeet = kHeads * DP * 4 <= kStage ? kHeads : 8;
  static constexpr int kORow = kMeet * (DP + 4) * 4 <= kStage ? DP + 4 : DP;
  static constexpr int kSmem = kRing + kQBytes;
  static constexpr int kTile = kWarps * kTok;                  // tokens of a CTA's tile
  static_assert(kMeet * kORow * 4 <= kStage, "a stage has to hold a warp's outputs");
  static_assert(kCtasPerSm * (kSmem + kStatic) <= 228 * 1024, "the CTAs of an SM have to fit its shared memory");
};

// 16-byte chunk c of row r, so that the eight rows of a matrix lie in different banks: as many bits of the row as its length leaves alike
// are exclusive-ored into the chunk's number (rows of 8, 4 or 2 chunks times an odd number start at 1, 2 or 4 places in the banks).
template <int kRow>
struct Swizzle {
  static constexpr int kMask = kRow % 128 == 0 ? 7 : (kRow % 64 == 0 ? 3 : 1), kShift = kMask == 7 ? 0 : (kMask == 3 ? 1 : 2);
  static __device__ __forceinline__ uint32_t bits(int r) { return (r >> kShift) & kMask; }
  static __device__ __forceinline__ uint32_t at(int r, int c) { return r * kRow + ((c ^ bits(r)) << 4); }
};

__device__ __forceinline__ int seq_len(const PagedAttnParams& p, int b) {
  const int32_t n = p.seqlens[b];
  return static_cast<int>(min(static_cast<int64_t>(n < 0 ? 0 : n), p.cap));
}

// ---- what is left when all CTAs of a unit are done: cut sequences are joined, scores become weights ----

template <int kThreads>      // among the kThreads threads that use this barrier
__device__ __forceinline__ void sync_threads(int barrier) { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(kThreads) : "memory"); }

__device__ __forceinline__ void join_pair(float& m, float& l, float om, float ol) {
  const float mn = fmaxf(m, om);
  l = mn == -INFINITY ? l + ol : l * ex2(m - mn) + ol * ex2(om - mn);      // (no references: no tokens, or no numbers)
  m = mn;
}

// This CTA's part of joining the sequence that is cut at the end of its run (tail: sequence or -1, its first and last run).  The CTAs of
// all runs but the last one that have tiles of the sequence share the join: each takes some of the outputs, four values of a head an item, and
// some threads an item, which take some of the pieces (slot 1 of the first run, slot 0 of the others).  At most four threads an item: more
// shorten the walk over the pieces by less than the exchange at its end takes (B = 1, 1001 tokens, in two kernels: 8.3 us with sixteen, 7.9 with
// four).
template <int kThreads>
__device__ __forceinline__ void join_tail(const PagedAttnParams& p, int tid, int barrier, int unit, int run, const int4& tail, float4* sums, float2* mls) {
  if (tail.x < 0) return;
  const int hk = unit / p.groups, h0 = (unit - hk * p.groups) * p.slots, nh = min(p.G - h0, p.slots);
  const int n = tail.z - tail.y + 1, helpers = n - 1, helper = run - tail.y;
  if (n < 2) return;
  const int Dv = p.c.Dv, vecs = Dv / 4, all = nh * vecs;
  const int item0 = all * helper / helpers, items = all * (helper + 1) / helpers - item0;
  if (items == 0) return;
  const int share = items >= kThreads ? 1 : min(min(kThreads / items, 4), n), at_once = kThreads / share;
  const int my = tid / share, part = tid - my * share;
  const int64_t out0 = static_cast<int64_t>(tail.x) * p.Hq + hk * p.G + h0;
  for (int base = 0; base < items; base += at_once) {
    const bool on = my < at_once && base + my < items;
    const int item = item0 + base + my, r = item / vecs, d = (item - r * vecs) * 4;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float m = -INFINITY, l = 0.0f;
    if (on) {                                  // maximum, sum and output together: one round trip to memory for four pieces
      constexpr int kPieces = 4;
      for (int i0 = part; i0 < n; i0 += share * kPieces) {
        float2 ml[kPieces];
        float4 x[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          const int i = i0 + k * share;
          if (i < n) {
            const int64_t s = ((static_cast<int64_t>(tail.y + i) * p.U + unit) * 2 + (i == 0 ? 1 : 0)) * p.part_rows + r;
            ml[k] = *reinterpret_cast<const float2*>(p.part_ml + s * 2);
            x[k] = *reinterpret_cast<const float4*>(p.part + s * Dv + d);
          }
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          if (i0 + k * share < n) {
            const float mn = fmaxf(m, ml[k].x);
            const float a = m == -INFINITY ? 0.0f : ex2(m - mn), w = ml[k].x == -INFINITY ? 0.0f : ex2(ml[k].x - mn);
            m = mn;
            l = l * a + ml[k].y * w;
            acc.x = acc.x * a + x[k].x * w;
            acc.y = acc.y * a + x[k].y * w;
            acc.z = acc.z * a + x[k].z * w;
            acc.w = acc.w * a + x[k].w * w;
          }
        }
      }
    }
    if (share > 1) {
      sync_threads<kThreads>(barrier);
      sums[tid] = acc;
      mls[tid] = make_float2(m, l);
      sync_threads<kThreads>(barrier);
    }
    if (on && part == 0) {
      if (share > 1) {
        for (int i = 1; i < share; ++i) m = fmaxf(m, mls[tid + i].x);
        l = 0.0f;
        acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int i = 0; i < share; ++i) {
          const float2 ml = mls[tid + i];
          const float w = ml.x == -INFINITY ? 0.0f : ex2(ml.x - m);
          const float4 x = sums[tid + i];
          l = fmaf(ml.y, w, l);
          acc.x = fmaf(x.x, w, acc.x);
          acc.y = fmaf(x.y, w, acc.y);
          acc.z = fmaf(x.z, w, acc.z);
          acc.w = fmaf(x.w, w, acc.w);
        }
      }
      const float inv = 1.0f / l;
      *reinterpret_cast<uint2*>(p.out + (out0 + r) * Dv + d) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      if (d == 0 && p.lse) p.lse[out0 + r] = (m + log2f(l * kUp)) * 0.6931471805599453f;
    }
  }
}

// Adds the weights of positions first + tid, first + tid + step ... below `end` of sequence b; span: the first and the last run that have tiles
// of it.  A block of threads, or a warp where no KV head has more than 8 query heads.  The first scores are asked for before the sums of the
// softmax that they wait for.
template <int kThreads>
__device__ __forceinline__ void add_weights(const PagedAttnParams& p, int tid, int b, int hk, int2 span, int first, int step, int end, float* lse2_sm) {
  constexpr int kAtOnce = kAtOnceWeights;
  const int64_t at = (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.score_ld + first + tid, score_step = static_cast<int64_t>(step) * p.score_heads;
  const float* s = p.scores + at * p.score_heads;
  float* out = p.weights + (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.ld + first + tid;
  const bool four = p.score_heads == 4;          // the ordinary number: one load a position
  int left = end - first - tid;
  float4 x[kAtOnce];
  float was[kAtOnce];
  auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (left <= i * step) break;
      was[i] = out[static_cast<int64_t>(i) * step];
      if (four) {
        x[i] = __ldcg(reinterpret_cast<const float4*>(s + i * score_step));
      } else {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(s + i * score_step));
        x[i] = make_float4(y.x, y.y, 0.0f, 0.0f);
      }
    }
  };
  fetch();
  // log2 of the sum of 2^score of head g, from pieces lane, lane + lanes, ...
  auto lse2 = [&](int g, int lane, int lanes) {
    if (span.x == span.y) return p.lse2[static_cast<int64_t>(b) * p.Hq + hk * p.G + g];
    const int unit = hk * p.groups + g / p.slots, r = g % p.slots;
    float m = -INFINITY, l = 0.0f;
    for (int i = lane; i <= span.y - span.x; i += lanes) {
      const int64_t slot = (static_cast<int64_t>(span.x + i) * p.U + unit) * 2 + (i == 0 ? 1 : 0);
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + (slot * p.part_rows + r) * 2);
      join_pair(m, l, ml.x, ml.y);
    }
    for (int d = lanes / 2; d > 0; d >>= 1) {
      const float om = __shfl_xor_sync(0xffffffffu, m, d), ol = __shfl_xor_sync(0xffffffffu, l, d);
      join_pair(m, l, om, ol);
    }
    return m + log2f(l * kUp);
  };
  if constexpr (kThreads == 32) {                // four lanes a head
    const float lg = lse2(min(tid >> 2, p.G - 1), tid & 3, 4);
    __syncwarp();
    if ((tid & 3) == 0) lse2_sm[tid >> 2] = lg;
    __syncwarp();
  } else {
    for (int g = tid >> 5; g < p.G; g += kThreads / 32) {
      const float lg = lse2(g, tid & 31, 32);
      if ((tid & 31) == 0) lse2_sm[g] = lg;
    }
    __syncthreads();
  }
  // (no weight for a head that is not there)
  const float l0 = lse2_sm[0], l1 = p.G > 1 ? lse2_sm[1] : INFINITY, l2 = four ? lse2_sm[2] : INFINITY, l3 = four && p.G > 3 ? lse2_sm[3] : INFINITY;
  while (left > 0) {
    float acc[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      acc[i] = ex2(x[i].x - l0) + (l1 != INFINITY ? ex2(x[i].y - l1) : 0.0f);
      if (four) acc[i] = acc[i] + ex2(x[i].z - l2) + (l3 != INFINITY ? ex2(x[i].w - l3) : 0.0f);
    }
    if (!four) {
      for (int g = 2; g < p.G; g += 2) {
        const float la = lse2_sm[g], lb = g + 1 < p.G ? lse2_sm[g + 1] : INFINITY;
        float2 y[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (left > i * step) y[i] = __ldcg(reinterpret_cast<const float2*>(s + i * score_step + g));
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (left > i * step) acc[i] += ex2(y[i].x - la) + (lb != INFINITY ? ex2(y[i].y - lb) : 0.0f);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      if (left > i * step) out[static_cast<int64_t>(i) * step] = was[i] + acc[i];
    left -= step * kAtOnce;
    s += score_step * kAtOnce;
    out += static_cast<int64_t>(step) * kAtOnce;
    fetch();
  }
}

// kJoin: the CTAs of a unit are a cluster, which joins its sequences and adds their weights itself.
template <bool kInt8, int DP, int kHeads, bool kJoin>
__global__ void __launch_bounds__((Shape<kInt8, DP, kHeads>::kThreads), (Shape<kInt8, DP, kHeads>::kCtasPerSm))
attn_paged_kernel(const __grid_constant__ PagedAttnParams p) {
  using S = Shape<kInt8, DP, kHeads>;
  constexpr int NT = kHeads / 8;                        // column tiles of heads
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ float ml[3][S::kWarps][kHeads];              // of a warp: references, sums, units of its outputs
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __shared__ int4 tail_sm;                               // (kJoin)
  // kJoin: the lengths, read once, so that all warps walk alike and meet at their barriers whatever becomes of the lengths meanwhile.  (Otherwise
  // a warp that is done leaves, and no barrier waits for it.)
  __shared__ int lengths[kJoin ? kClusterTiles * kClusterCtas : 1];
  const int unit = kJoin ? blockIdx.x / p.runs : blockIdx.x % p.U, run = kJoin ? blockIdx.x % p.runs : blockIdx.x / p.U;
  const int hk = unit / p.groups, h0 = (unit - hk * p.groups) * kHeads;        // first head of the group within the KV head
  const int nh = min(p.G - h0, kHeads);
  const int64_t head0 = static_cast<int64_t>(hk) * p.G + h0;

  pdl_wait_primary();
  pdl_launch_dependents();

  // ---- this CTA's run of tiles ----  (every warp by itself; a lane looks at a share of the sequences)
  if constexpr (kJoin) {
    for (int b = threadIdx.x; b < p.B; b += S::kThreads) lengths[b] = seq_len(p, b);
    __syncthreads();
  }
  auto len_of = [&](int b) { return kJoin ? lengths[b] : seq_len(p, b); };
  const int per_lane = (p.B + 31) / 32, b_lo = min(p.B, lane * per_lane), b_hi = min(p.B, b_lo + per_lane);
  int mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const int L = len_of(b);
    if (warp == 0) {
      if (blockIdx.x == 0 && L != p.seqlens[b]) atomicMax(p.status, kStatusBadShape);
      if (L == 0 && b % p.runs == run) {         // nothing to attend to
        for (int h = 0; h < nh; ++h) {
          const int64_t out_row = static_cast<int64_t>(b) * p.Hq + head0 + h;
          for (int d = 0; d < p.c.Dv; d += 8) *reinterpret_cast<uint4*>(p.out + out_row * p.c.Dv + d) = make_uint4(0, 0, 0, 0);
          if (p.lse) p.lse[out_row] = -INFINITY;
        }
      }
    }
    mine += (L + S::kTile - 1) / S::kTile;
  }
  int before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, before, d);
    if (lane >= d) before += y;
  }
  const int T = __shfl_sync(0xffffffffu, before, 31);
  before -= mine;
  int4* tail = kJoin ? &tail_sm : p.tail + blockIdx.x;
  if (threadIdx.x == 0) *tail = make_int4(-1, 0, 0, 0);
  const int runs = min(p.runs, T);                // (no empty runs)
  auto meet_cluster = [&]() {                     // every CTA of the unit is done; the rings are free
    cluster_arrive_all();
    cluster_wait_all();
    float4* sums = reinterpret_cast<float4*>(smem);
    float2* mls = reinterpret_cast<float2*>(sums + S::kThreads);
    float* lse2_sm = reinterpret_cast<float*>(mls + S::kThreads);
    constexpr int kHalf = S::kThreads / 2;        // half of the warps join while the others add weights
    if (threadIdx.x < kHalf) join_tail<kHalf>(p, threadIdx.x, 1, unit, run, tail_sm, sums, mls);
    if (threadIdx.x < kHalf || !p.weights) return;
    // (blocks of positions, dealt out in turn to the warps of all CTAs, sequence after sequence)
    constexpr int kBlock = 32 * kAtOnceWeights, kAdders = S::kWarps - S::kWarps / 2;
    const int adders = p.runs * kAdders, adder = run * kAdders + warp - S::kWarps / 2;
    lse2_sm += warp * 8;
    int at = 0, turn = adder;                     // tiles of the sequences before this one; this warp's first block of it
    for (int b = 0; b < p.B; ++b) {
      const int L = lengths[b], upto = at + (L + S::kTile - 1) / S::kTile;
      for (; turn * kBlock < L; turn += adders) {
        // (there are few tiles: 32 bits will do)
        const int2 span = make_int2(((at + 1) * runs - 1) / T, min((upto * runs - 1) / T, runs - 1));
        add_weights<32>(p, lane, b, hk, span, turn * kBlock, 32, min(L, (turn + 1) * kBlock), lse2_sm);
      }
      turn -= (L + kBlock - 1) / kBlock;
      at = upto;
    }
  };
  if (run >= runs) {
    if constexpr (kJoin) meet_cluster();
    return;
  }
  auto run_start = [&](int r) { return static_cast<int>(static_cast<int64_t>(r) * T / runs); };
  const int first = run_start(run), end = run_start(run + 1);
  const bool here = first >= before && first < before + mine;       // of one lane
  int b_first = b_lo, t_first = first - before;
  if (here) {
    for (; b_first + 1 < b_hi; ++b_first) {
      const int t = (len_of(b_first) + S::kTile - 1) / S::kTile;
      if (t_first < t) break;
      t_first -= t;
    }
  }
  const int owner = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
  b_first = __shfl_sync(0xffffffffu, b_first, owner);
  t_first = __shfl_sync(0xffffffffu, t_first, owner);

  // A walk over the tiles of the run, one for the loads and one for the arithmetic.
  struct Walk {
    int b, tile, tiles, L, left;          // sequence, tile of it, tiles of it, its length, tiles left in the run
  };
  Walk ld;
  ld.b = b_first;
  ld.tile = t_first;
  ld.L = len_of(ld.b);
  ld.tiles = (ld.L + S::kTile - 1) / S::kTile;
  ld.left = end - first;
  Walk cur = ld;
  auto next_sequence = [&](Walk& w) {
    do {                                      // (there is one, unless the lengths are changed meanwhile)
      w.b = min(w.b + 1, p.B - 1);
      w.L = len_of(w.b);
    } while (w.L == 0 && w.b + 1 < p.B);
    w.tile = 0;
    w.tiles = (w.L + S::kTile - 1) / S::kTile;
  };

  // ---- loads ----
  const uint64_t policy = p.leave_l2 ? policy_evict_first() : policy_evict_normal();
  uint8_t* ring = smem + warp * (S::kStages * S::kStage);
  const uint32_t ring_u = smem_u32(ring);
  using W = Swizzle<S::kRow>;
  constexpr int kChunks = S::kRow / 16;                 // 16-byte chunks of a row
  constexpr int kLanes = kChunks <= 4 ? 4 : (kChunks <= 8 ? 8 : (kChunks <= 16 ? 16 : 32));      // lanes that bring a row, some of them idle
  constexpr int kRowsPer = 32 / kLanes;                 // rows that one instruction of the warp brings
  const int my_chunk = lane % kLanes, my_row = lane / kLanes;
  const bool busy = kLanes == kChunks || my_chunk < kChunks;
  const uint8_t* kbase = p.c.k.base + hk * p.c.k.head + my_chunk * 16;
  const uint8_t* vbase = p.c.v.base + hk * p.c.v.head + my_chunk * 16;
  const uint8_t* ksbase = kInt8 ? p.c.ks.base + hk * p.c.ks.head : nullptr;
  const uint8_t* vsbase = kInt8 ? p.c.vs.base + hk * p.c.vs.head : nullptr;
  const bool k_there = my_chunk * 16 < p.c.D * S::kEs, v_there = my_chunk * 16 < p.c.Dv * S::kEs;
  // Instruction i brings row i * kRowsPer + my_row to the lanes of my_row.  The lane that looks that row up is the i-th of them, so that
  // the others get its offset by a shuffle whose index is a constant.
  constexpr int kIter = S::kTok / kRowsPer;
  const int tok_lane = my_chunk % kIter * kRowsPer + my_row;
  const uint32_t lane_dst = W::at(my_row, my_chunk);
  // The block of this lane's token of the tile that `ld` stands on, asked for a tile ahead; -1 behind the end.
  const int32_t* ld_table = p.table + static_cast<int64_t>(ld.b) * p.max_blocks;
  int ld_pos = ld.tile * S::kTile + warp * S::kTok + tok_lane;
  uint32_t ld_page = 0;
  int blk = -1;
  auto look_up = [&]() {
    blk = -1;
    if (ld_pos < ld.L) {
      ld_page = div_by(ld_pos, p.c.page);
      blk = ld_table[ld_page];
    }
  };
  look_up();
  auto issue = [&](uint32_t dst) {
    if (ld.left > 0) {
      const bool wanted = ld_pos < ld.L;
      const bool there = wanted && static_cast<uint32_t>(blk) < static_cast<uint32_t>(p.c.num_blocks);
      if (wanted && !there) atomicMax(p.status, kStatusBadShape);
      const uint32_t slot = ld_pos - ld_page * p.c.page.d, at = there ? blk : 0;
      const uint32_t in = there ? slot : 0;
      const uint32_t ko = at * p.k_block + in * p.k_token, vo = at * p.v_block + in * p.v_token;
      const uint32_t mask = __ballot_sync(0xffffffffu, there);
      const uint32_t at_k = dst + lane_dst, at_v = at_k + S::kHalf;
      auto to = [&](uint32_t base, int i) { return (base ^ (W::bits(i * kRowsPer) << 4)) + i * kRowsPer * S::kRow; };
      auto from = [&](const uint8_t* base, uint32_t off, int i) { return base + static_cast<uint64_t>(__shfl_sync(0xffffffffu, off, i, kLanes)) * 16; };
      if (__all_sync(0xffffffffu, mask == 0xffffffffu && ((k_there && v_there) || !busy))) {
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          const uint8_t* src = from(kbase, ko, i);
          if (busy) cp16_all(to(at_k, i), src, policy);
        }
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          const uint8_t* src = from(vbase, vo, i);
          if (busy) cp16_all(to(at_v, i), src, policy);
        }
      } else {                                          // zeros for rows behind the end and for values that a row does not have
        const uint32_t mine = mask >> (my_row * kLanes), k_mask = k_there ? mine : 0u, v_mask = v_there ? mine : 0u;
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          const uint8_t* src = from(kbase, ko, i);
          if (busy) cp16(to(at_k, i), src, (k_mask >> i) & 1u, policy);
        }
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          const uint8_t* src = from(vbase, vo, i);
          if (busy) cp16(to(at_v, i), src, (v_mask >> i) & 1u, policy);
        }
      }
      if constexpr (kInt8) {
        const uint32_t sc = dst + 2 * S::kHalf + tok_lane * 4;
        const uint32_t kso = at * p.ks_block + in * p.ks_token, vso = at * p.vs_block + in * p.vs_token;
        if (S::kTok == 32 || my_chunk < kIter) cp4(sc, ksbase + static_cast<uint64_t>(kso) * 4, there);
        if (S::kTok == 32 || my_chunk >= kIter) cp4(sc + S::kScale, vsbase + static_cast<uint64_t>(vso) * 4, there);
      }
      --ld.left;
      ld_pos += S::kTile;
      if (++ld.tile == ld.tiles && ld.left > 0) {
        next_sequence(ld);
        ld_table = p.table + static_cast<int64_t>(ld.b) * p.max_blocks;
        ld_pos = warp * S::kTok + tok_lane;
      }
      look_up();
    }
    cp_commit();
  };
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) issue(ring_u + s * S::kStage);

  // ---- the arithmetic ----
  const int row = lane >> 2, quad = lane & 3;           // a thread has tokens (or values of d) `row`, `row` + 8 and heads 2 quad, 2 quad + 1
  uint2* sm_q = reinterpret_cast<uint2*>(smem + S::kRing);
  __shared__ uint32_t q_big[S::kQInSmem && kInt8 ? S::kWarps : 1][kHeads];
  constexpr int kSteps = DP / 16;
  uint2 qf[S::kQInSmem ? 1 : kSteps][NT];
  float o[NT][DP / 16][4];
  float m[NT][2], l[NT][2], f[NT][2];                   // f: from products to log2 scores
  const int k_steps = (p.c.D + 15) / 16, v_steps = (p.c.Dv + 15) / 16;

  // The query as column fragments: head `row` of each tile.  INT8: of 16 values of d a thread's bytes are 4 quad ... 4 quad + 3, so the
  // query is taken in that order too, and goes into FP16 scaled by a power of two that brings its largest value to 2^14 ... 2^15: what
  // is 2^-29 of that or more stays exact, the rest is off by 2^-40 of it at most.
  auto raw_q = [&](int s, int n) {
    const uint16_t* q = p.q + static_cast<int64_t>(cur.b) * p.q_ld + head0 * p.c.D;
    uint2 v = make_uint2(0, 0);
    const int h = n * 8 + row;
    const uint16_t* at = q + h * p.c.D + s * 16;
    if (h < nh) {
      if constexpr (kInt8) {
        if (s * 16 + 4 * quad < p.c.D) v = *reinterpret_cast<const uint2*>(at + 4 * quad);
      } else {
        if (s * 16 + 2 * quad < p.c.D) v.x = *reinterpret_cast<const uint32_t*>(at + 2 * quad);
        if (s * 16 + 2 * quad + 8 < p.c.D) v.y = *reinterpret_cast<const uint32_t*>(at + 2 * quad + 8);
      }
    }
    return v;
  };
  auto fetch_q = [&]() {       // (of the sequence that `cur` stands on)
    if constexpr (!S::kQInSmem) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) qf[s][n] = raw_q(s, n);
      }
    }
  };
  auto ready_q = [&]() {
    // In shared memory: each warp brings some of the steps, kMine at most, all its loads under way together, and the warps tell each other the largest
    // values (each warp looking at every step: 128 / 8 heads of 256, 40 x 1000-2000 tokens INT8 100 -> 74 us, BF16 106 -> 99).
    constexpr int kMine = S::kQInSmem ? (kSteps + S::kWarps - 1) / S::kWarps : kSteps;
    uint2 mine[S::kQInSmem ? kMine : 1][NT];
    if constexpr (S::kQInSmem) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
#pragma unroll
        for (int n = 0; n < NT; ++n) mine[i][n] = raw_q(warp + i * S::kWarps, n);
      }
    }
    float up[NT];
    if constexpr (kInt8) {
      uint32_t big[NT];                                 // of |x| as BF16 bits, which grow with the value
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        big[n] = 0;
#pragma unroll
        for (int s = 0; s < kMine; ++s) {
          const uint2 v = S::kQInSmem ? mine[S::kQInSmem ? s : 0][n] : qf[S::kQInSmem ? 0 : s][n];
          big[n] = __vmaxu2(big[n], __vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu));
        }
        big[n] = max(big[n] & 0xFFFFu, big[n] >> 16);
        big[n] = max(big[n], __shfl_xor_sync(0xffffffffu, big[n], 1));
        big[n] = max(big[n], __shfl_xor_sync(0xffffffffu, big[n], 2));
      }
      if constexpr (S::kQInSmem) {                      // of all warps' steps
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (quad == 0) q_big[warp][n * 8 + row] = big[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int w = 0; w < S::kWarps; ++w) big[n] = max(big[n], q_big[w][n * 8 + row]);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // the exponent of the largest value, from -126 (or less: taken as that) to 127
        const int e = max(static_cast<int>(big[n] >> 7), 1) - 127;
        // 2^(14 - e), cut to what a float holds: then the values are small, and stay exact as well
        up[n] = __uint_as_float(static_cast<uint32_t>(min(14 - e, 126) + 127) << 23);
        const float down = p.scale2 / up[n];
        f[n][0] = __shfl_sync(0xffffffffu, down, 8 * quad);
        f[n][1] = __shfl_sync(0xffffffffu, down, 8 * quad + 4);
      }
    }
    auto fragment = [&](uint2 v, int n) {
      if constexpr (kInt8) {
        return make_uint2(pack_f16(__uint_as_float(v.x << 16) * up[n], __uint_as_float(v.x & 0xFFFF0000u) * up[n]),
                          pack_f16(__uint_as_float(v.y << 16) * up[n], __uint_as_float(v.y & 0xFFFF0000u) * up[n]));
      } else {
        return v;
      }
    };
    if constexpr (S::kQInSmem) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int s = warp + i * S::kWarps;
        if (s < kSteps) {
#pragma unroll
          for (int n = 0; n < NT; ++n) sm_q[(s * NT + n) * 32 + lane] = fragment(mine[i][n], n);
        }
      }
      __syncthreads();
    } else if constexpr (kInt8) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) qf[s][n] = fragment(qf[s][n], n);
      }
    }
  };
  auto q_fragment = [&](int s, int n) {
    if constexpr (S::kQInSmem) return sm_q[(s * NT + n) * 32 + lane];
    else return qf[s][n];
  };
#pragma unroll
  for (int n = 0; n < NT; ++n) f[n][0] = f[n][1] = p.scale2;

  // Matrices of the fragments: token (lane & 15) of 16, chunks c and c + 1 by the upper half of the warp; BF16 values: tokens by the upper
  // half, chunks by the eighths.  The swizzle moves only the lowest bits of a chunk's number, so
  // chunk c is an exclusive or away from chunk 0, and what lies above those bits an offset.
  const uint32_t k_lane = W::at(lane & 15, lane >> 4);
  const uint32_t v_lane = S::kHalf + (kInt8 ? k_lane : W::at(((lane >> 4) << 3) + (lane & 7), (lane >> 3) & 1));
  constexpr int kSwz = W::kMask;
  uint32_t stage_u = ring_u, fill_u = ring_u + (S::kStages - 1) * S::kStage;      // the stage of this tile, and the one to fill
  const float* stage_scales = reinterpret_cast<const float*>(ring + 2 * S::kHalf);
  fetch_q();
  while (cur.left > 0) {
    // a segment: the tiles of one sequence that are in this run
    const int seg_first = cur.tile;
    const int seg = min(cur.tiles - cur.tile, cur.left);
    const int b = cur.b, L = cur.L;
    ready_q();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.0f;
    }
    // INT8: vref, a power of two that no value's scale so far exceeds (2^-111 at least, so that vinv is finite).  P times the scale is in
    // units of vref / 2^7: at most 2^15 in FP16, 11 bits down to 2^-21 vref, off by 2^-32 vref below that.
    float vref = 3.851859888774472e-34f, vinv = kPUnits / vref;

    float* score_at = nullptr;
    if (p.weights)
      score_at = p.scores + ((static_cast<int64_t>(b) * p.c.Hkv + hk) * p.score_ld + warp * S::kTok + row) * p.score_heads + h0 + 2 * quad;
    for (int t = 0; t < seg; ++t) {
      cp_wait<S::kStages - 2>();
      __syncwarp();
      issue(fill_u);                                    // the stage that the last tile left
      const uint32_t k_u = stage_u + k_lane, v_u = stage_u + v_lane;
      const float* scales = stage_scales;
      fill_u = stage_u;
      stage_u += S::kStage;
      stage_scales += S::kStage / 4;
      if (stage_u == ring_u + S::kStages * S::kStage) {
        stage_u = ring_u;
        stage_scales -= S::kStages * S::kStage / 4;
      }
      const int tile = seg_first + t, pos0 = tile * S::kTile + warp * S::kTok;
      if (pos0 >= L) continue;                          // (uniform in the warp)
      constexpr int kGroups = S::kTok / 16;

      // scores of 16 tokens (rows) and 8 heads (columns) a fragment
      float s[kGroups][NT][4];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
#pragma unroll
        for (int c4 = 0; c4 < kSteps; c4 += 4) {        // 64 values of d at a time: what is past D is zero in both
          if (c4 >= k_steps) break;
#pragma unroll
          for (int c = c4; c < c4 + 4 && c < kSteps; c += kInt8 ? 2 : 1) {
            uint32_t r[4];
            const int chunk = kInt8 ? c : 2 * c;
            ldsm4(r, (k_u ^ ((chunk & kSwz) << 4)) + ((chunk & ~kSwz) << 4) + g * 16 * S::kRow);
            if constexpr (kInt8) {                      // a register: four codes of a token; two registers a step
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const uint32_t x = r[2 * j] ^ 0x80808080u, y = r[2 * j + 1] ^ 0x80808080u;
                const uint32_t a[4] = {codes_f16<0, 1>(x), codes_f16<0, 1>(y), codes_f16<2, 3>(x), codes_f16<2, 3>(y)};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  if (c + j == 0) mma16<true, true>(s[g][n], a, q_fragment(0, n));
                  else mma16<true>(s[g][n], a, q_fragment(c + j, n));
                }
              }
            } else {
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                if (c == 0) mma16<false, true>(s[g][n], r, q_fragment(0, n));
                else mma16<false>(s[g][n], r, q_fragment(c, n));
              }
            }
          }
        }
      }
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        float k0 = 1.0f, k1 = 1.0f;
        if constexpr (kInt8) {
          k0 = scales[g * 16 + row];
          k1 = scales[g * 16 + row + 8];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[g][n][e] *= f[n][e] * k0;
            s[g][n][2 + e] *= f[n][e] * k1;
          }
        }
      }
      const int left = L - pos0 - row;                  // tokens from this thread's first one on
      if (pos0 + S::kTok > L) {                         // (uniform) the sequence ends in this tile
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if (left <= g * 16) s[g][n][e] = -INFINITY;
              if (left <= g * 16 + 8) s[g][n][2 + e] = -INFINITY;
            }
          }
        }
      }
      if (p.weights) {
        float* dst = score_at + static_cast<int64_t>(tile) * (S::kTile * p.score_heads);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if (n * 8 + 2 * quad < nh) {
              if (left > g * 16) *reinterpret_cast<float2*>(dst + (g * 16) * p.score_heads + n * 8) = make_float2(s[g][n][0], s[g][n][1]);
              if (left > g * 16 + 8) *reinterpret_cast<float2*>(dst + (g * 16 + 8) * p.score_heads + n * 8) = make_float2(s[g][n][2], s[g][n][3]);
            }
          }
        }
      }

      // Softmax.  The reference of a head moves only when a score exceeds it by more than 2^8 (it cancels in the end; probabilities up to
      // 2^8 cost nothing in FP32), which after the first tile is rare, and only then do the lanes ask each other for the maximum.
      float mx[NT][2];
      bool moved = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[n][e] = fmaxf(s[0][n][e], s[0][n][2 + e]);
#pragma unroll
          for (int g = 1; g < kGroups; ++g) mx[n][e] = fmaxf(mx[n][e], fmaxf(s[g][n][e], s[g][n][2 + e]));
          moved = moved || mx[n][e] > m[n][e] + kHeld;
        }
      }
      float vs[kGroups][2];
      float vnew = vref;
      if constexpr (kInt8) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(scales[S::kTok + (lane & (S::kTok - 1))]) & 0x7FFFFFFFu);
        if (top > __float_as_uint(vref)) {              // (uniform) the next power of two
          vnew = __uint_as_float(min((top + 0x007FFFFFu) & 0x7F800000u, 0x7F000000u));
          moved = true;
        }
      }
      if (__any_sync(0xffffffffu, moved)) {
        const float vr = kInt8 ? vref / vnew : 1.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) mx[n][e] = fmaxf(mx[n][e], __shfl_xor_sync(0xffffffffu, mx[n][e], d));
            mx[n][e] = fmaxf(mx[n][e], m[n][e]);
            const float r = mx[n][e] == -INFINITY ? 1.0f : ex2(m[n][e] - mx[n][e]);
            m[n][e] = mx[n][e];
            l[n][e] *= r;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
              o[n][i][e] *= r * vr;
              o[n][i][2 + e] *= r * vr;
            }
          }
        }
        if constexpr (kInt8) {
          vref = vnew;
          vinv = kPUnits / vnew;
        }
      }
      if constexpr (kInt8) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          vs[g][0] = scales[S::kTok + g * 16 + row] * vinv;
          vs[g][1] = scales[S::kTok + g * 16 + row + 8] * vinv;
        }
      }
      // Probabilities as column fragments of the product with v: the transposes of the score fragments.  INT8: times the value's scale,
      // in FP16 (11 bits).  BF16: the 8 bits of one BF16 would double the error of the result, so what they leave out goes in too.  They are
      // cut off, not rounded, and the last bit of P is set, so that what is left out is above 0: at most 2^-7 of P, rounded to 8 bits (2^-16).
      uint2 ph[kGroups][NT], pl[kGroups][NT];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float mm = m[n][e & 1];
            x[e] = ex2(s[g][n][e] - (mm == -INFINITY ? 0.0f : mm));
            if constexpr (!kInt8) x[e] = __uint_as_float(__float_as_uint(x[e] * kDown) | 1u);
            l[n][e & 1] += x[e];
          }
          if constexpr (kInt8) {
            ph[g][n] = make_uint2(transposed(pack_f16(x[0] * vs[g][0], x[1] * vs[g][0])), transposed(pack_f16(x[2] * vs[g][1], x[3] * vs[g][1])));
          } else {
            const uint32_t a = high_halves(x[0], x[1]), c = high_halves(x[2], x[3]);
            ph[g][n] = make_uint2(transposed(a), transposed(c));
            pl[g][n] = make_uint2(transposed(pack_bf16(x[0] - __uint_as_float(a << 16), x[1] - __uint_as_float(a & 0xFFFF0000u))),
                                  transposed(pack_bf16(x[2] - __uint_as_float(c << 16), x[3] - __uint_as_float(c & 0xFFFF0000u))));
          }
        }
      }
      // 16 values of d (rows) and 8 heads a fragment
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
#pragma unroll
        for (int c4 = 0; c4 < DP / 16; c4 += 4) {
          if (c4 >= v_steps) break;
#pragma unroll
          for (int c = c4; c < c4 + 4 && c < kSteps; c += kInt8 ? 2 : 1) {
            uint32_t r[4];
            const int chunk = kInt8 ? c : 2 * c;
            ldsm4_t(r, (v_u ^ ((chunk & kSwz) << 4)) + ((chunk & ~kSwz) << 4) + g * 16 * S::kRow);
            if constexpr (kInt8) {                      // a register: two tokens of an even and the next odd value of d
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const uint32_t x = r[2 * j] ^ 0x80808080u, y = r[2 * j + 1] ^ 0x80808080u;
                const uint32_t a[4] = {codes_f16<0, 2>(x), codes_f16<1, 3>(x), codes_f16<0, 2>(y), codes_f16<1, 3>(y)};
#pragma unroll
                for (int n = 0; n < NT; ++n) mma16<true>(o[n][c + j], a, ph[g][n]);
              }
            } else {
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                mma16<false>(o[n][c], r, ph[g][n]);
                mma16<false>(o[n][c], r, pl[g][n]);
              }
            }
          }
        }
      }
    }
    cur.left -= seg;
    if (cur.left > 0) {                                 // (a segment that is not the run's last one ends its sequence)
      next_sequence(cur);
      fetch_q();
    }

    // ---- the segment's end: the warps meet ----
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
        if (row == 0) {
          const int h = n * 8 + 2 * quad + e;
          ml[0][warp][h] = m[n][e];
          ml[1][warp][h] = kInt8 ? l[n][e] * kDown : l[n][e];
          if constexpr (kInt8) ml[2][warp][h] = vref * (1.0f / kPUnits);
        }
      }
    }
    const bool from_start = seg_first == 0, to_end = seg_first + seg == (L + S::kTile - 1) / S::kTile;
    const int Dv = p.c.Dv, vecs = Dv / 4;
    const int64_t slot = (kJoin ? static_cast<int64_t>(run) * p.U + unit : static_cast<int64_t>(blockIdx.x)) * 2 + (from_start ? 1 : 0);
    float* meet = reinterpret_cast<float*>(smem + (fill_u - smem_u32(smem)));      // this warp's stage; the others' are as far from their rings
#pragma unroll
    for (int pass = 0; pass < kHeads / S::kMeet; ++pass) {
#pragma unroll
      for (int n = pass * (S::kMeet / 8); n < (pass + 1) * (S::kMeet / 8); ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (n * 8 + 2 * quad + e < nh) {
            float* dst = meet + (n * 8 + 2 * quad + e - pass * S::kMeet) * S::kORow;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
              if constexpr (kInt8) {
                *reinterpret_cast<float2*>(dst + i * 16 + 2 * row) = make_float2(o[n][i][e] * kDown, o[n][i][2 + e] * kDown);
              } else {
                dst[i * 16 + row] = o[n][i][e];
                dst[i * 16 + row + 8] = o[n][i][2 + e];
              }
            }
          }
        }
      }
      __syncthreads();
      const float* met = reinterpret_cast<const float*>(smem + (fill_u - ring_u));      // warp 0's; the next one's is a ring further
      const int heads = min(nh - pass * S::kMeet, S::kMeet);
      for (int i = threadIdx.x; i < heads * vecs; i += S::kThreads) {
        const int hl = i / vecs, d = (i - hl * vecs) * 4, h = pass * S::kMeet + hl;
        float mh = ml[0][0][h];
#pragma unroll
        for (int w = 1; w < S::kWarps; ++w) mh = fmaxf(mh, ml[0][w][h]);
        float lh = 0.0f;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < S::kWarps; ++w) {              // (a fixed order)
          const float mw = ml[0][w][h];
          // (a warp without a reference has seen no token, or none whose score is a number: then its sum is none either, and goes on)
          const float r = mw == -INFINITY ? 0.0f : ex2(mw - mh), u = kInt8 ? r * ml[2][w][h] : r;
          const float4 x = *reinterpret_cast<const float4*>(met + w * (S::kStages * S::kStage / 4) + hl * S::kORow + d);
          lh = fmaf(ml[1][w][h], r, lh);
          v.x = fmaf(x.x, u, v.x);
          v.y = fmaf(x.y, u, v.y);
          v.z = fmaf(x.z, u, v.z);
          v.w = fmaf(x.w, u, v.w);
        }
        if (from_start && to_end) {
          const float inv = 1.0f / lh;
          const int64_t out_row = static_cast<int64_t>(b) * p.Hq + head0 + h;
          *reinterpret_cast<uint2*>(p.out + out_row * Dv + d) = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
          if (d == 0) {
            const float lg = mh + log2f(lh * kUp);
            if (p.lse) p.lse[out_row] = lg * 0.6931471805599453f;
            if (p.weights) p.lse2[out_row] = lg;
          }
        } else {
          *reinterpret_cast<float4*>(p.part + (slot * p.part_rows + h) * Dv + d) = v;
          if (d == 0) *reinterpret_cast<float2*>(p.part_ml + (slot * p.part_rows + h) * 2) = make_float2(mh, lh);
        }
      }
      __syncthreads();
    }
    if (threadIdx.x == 0) {                      // the runs that have tiles of this sequence
      const int64_t at = static_cast<int64_t>(end) - cur.left - seg - seg_first, upto = at + (L + S::kTile - 1) / S::kTile;
      // (between 0 and runs - 1, and apart where the sequence is cut, unless the lengths are changed meanwhile)
      const int run0 = max(static_cast<int>(((at + 1) * runs - 1) / T), 0), run1 = min(static_cast<int>((upto * runs - 1) / T), runs - 1);
      if (!kJoin && from_start && unit == 0) p.seq_runs[b] = make_int2(run0, run1);
      if (!to_end) *tail = make_int4(b, run0, run1, 0);
    }
  }
  cp_wait<0>();
  if constexpr (kJoin) meet_cluster();
}

// Joins the partial results of cut sequences (CTAs [0, runs x U), those whose run ends inside one), and adds the attention weights
// (the other CTAs: (sequence, KV head) x share of the positions) from the scores that the first kernel left.
__global__ void __launch_bounds__(kJoinThreads)
attn_paged_join_kernel(const __grid_constant__ PagedAttnParams p) {
  __shared__ float4 sums[kJoinThreads];
  __shared__ float2 mls[kJoinThreads];
  extern __shared__ float lse2_sm[];             // [G]
  pdl_wait_primary();
  pdl_launch_dependents();
  const int join_ctas = p.runs * p.U;
  if (static_cast<int>(blockIdx.x) < join_ctas) {
    join_tail<kJoinThreads>(p, threadIdx.x, 0, blockIdx.x % p.U, blockIdx.x / p.U, p.tail[blockIdx.x], sums, mls);
    return;
  }
  const int w = blockIdx.x - join_ctas, share = w % p.join_weight_ctas, bk = w / p.join_weight_ctas;
  const int b = bk / p.c.Hkv, hk = bk - b * p.c.Hkv;
  int2 span = p.seq_runs[b];                     // (anything at all for an empty sequence, and for one that has just stopped being one)
  span = make_int2(max(span.x, 0), min(span.y, p.runs - 1));
  const int L = seq_len(p, b);
  if (static_cast<int64_t>(share) * kJoinThreads >= L) return;
  add_weights<kJoinThreads>(p, threadIdx.x, b, hk, span, share * kJoinThreads, p.join_weight_ctas * kJoinThreads, L, lse2_sm);
}

struct PagedPlan {
  int slots, groups, U, runs, part_rows, score_heads;
  size_t part, ml, tail, seq_runs, lse2, scores, bytes;     // offsets into the workspace
};

// Head slots of a CTA: 8 for up to 8 query heads of a KV head, else 16, or 24 where that makes fewer groups of them and rows are not too wide for
// its registers (each group reads the cache and converts it: 160 / 8 heads of 128, 32 x 2048-8192 tokens BF16 188 -> 128 us, INT8
// 156 -> 107; of 192 280 -> 191, 232 -> 197).
int head_slots(int G, int widest) {
  if (G <= 8) return 8;
  return widest <= 192 && (G + 23) / 24 < (G + 15) / 16 ? 24 : 16;
}

// (ctas_per_sm: 4, the most of any kernel, where the head dimension is not known; the workspace has room for that)
bool plan_paged(int B, int Hq, int Hkv, int Dv, int64_t ld, int slots, int ctas_per_sm, PagedPlan* pl) {
  if (B < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hq > 8192 || B > (1 << 20) || Dv < 1 || Dv > 256 || ld < 0 || ld > 0x7FFFFFFF) return false;
  if (static_cast<int64_t>(B) * Hkv > (1 << 24) || static_cast<double>(B) * (Hq + Hkv) * ld > 1e15) return false;      // (grids and sizes that count)
  const int G = Hq / Hkv;
  pl->slots = slots;
  pl->groups = (G + pl->slots - 1) / pl->slots;
  pl->U = Hkv * pl->groups;
  pl->runs = sm_count() * ctas_per_sm / pl->U;
  if (pl->runs < 1) pl->runs = 1;
  pl->part_rows = G < pl->slots ? G : pl->slots;
  pl->score_heads = (G + 1) / 2 * 2;
  const size_t ctas = static_cast<size_t>(pl->runs) * pl->U;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = round_up(at + bytes, 256);
    return o;
  };
  pl->part = take(ctas * 2 * pl->part_rows * Dv * 4);
  pl->ml = take(ctas * 2 * pl->part_rows * 8);
  pl->tail = take(ctas * sizeof(int4));
  pl->seq_runs = take(static_cast<size_t>(B) * sizeof(int2));
  pl->lse2 = take(static_cast<size_t>(B) * Hq * 4);
  pl->scores = take(static_cast<size_t>(B) * Hkv * ld * pl->score_heads * 4);
  pl->bytes = round_up(at, 1024);
  return true;
}

template <bool kInt8, int DP, int kHeads, bool kJoin>
bool launch_runs(const PagedAttnParams& p, cudaStream_t s, bool pdl) {
  using Sh = Shape<kInt8, DP, kHeads>;
  auto kernel = attn_paged_kernel<kInt8, DP, kHeads, kJoin>;
  static DeviceOnce once;
  if (!once([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem) == cudaSuccess &&
               (!kJoin || cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess);
      }))
    return false;
  if (launch_pdl_cluster(kernel, dim3(p.runs * p.U), dim3(Sh::kThreads), Sh::kSmem, s, pdl, kJoin ? p.runs : 1, p) == cudaSuccess) return true;
  cudaGetLastError();
  return false;
}

template <bool kInt8, int DP, int kHeads>
msd_status_t launch_paged(const PagedAttnParams& p, bool cluster, cudaStream_t s) {
  const bool pdl = option(OPT_NO_PDL) != 1;
  if constexpr (kHeads == 8) {
    // (clusters of more than 8 CTAs are not promised by every device or part of one: without them two kernels do, with as many runs)
    if (cluster && option(OPT_ATTN_CLUSTER) != 0 && launch_runs<kInt8, DP, kHeads, true>(p, s, pdl)) return MSD_OK;
  }
  if (!launch_runs<kInt8, DP, kHeads, false>(p, s, pdl)) return MSD_ERR_CUDA;
  if (p.runs == 1 && !p.weights) return MSD_OK;      // (every sequence was finished by one CTA)
  const unsigned weight_ctas = p.weights ? static_cast<unsigned>(p.B) * p.c.Hkv * p.join_weight_ctas : 0;
  if (launch_pdl(attn_paged_join_kernel, dim3(p.runs * p.U + weight_ctas), dim3(kJoinThreads), p.weights ? p.G * sizeof(float) : 0, s, pdl, p) !=
      cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }
  return MSD_OK;
}

// f(kernel shape) for the shape of a call
template <typename F>
auto with_shape(bool int8, int widest, int slots, F&& f) {
  auto heads = [&](auto i8, auto dp) {
    if constexpr (decltype(dp)::value <= 192) {
      if (slots == 24) return f.template operator()<decltype(i8)::value, decltype(dp)::value, 24>();
    }
    return slots == 8 ? f.template operator()<decltype(i8)::value, decltype(dp)::value, 8>() : f.template operator()<decltype(i8)::value, decltype(dp)::value, 16>();
  };
  auto size = [&](auto i8) {
    if (widest <= 64) return heads(i8, std::integral_constant<int, 64>{});
    if (widest <= 96) return heads(i8, std::integral_constant<int, 96>{});
    if (widest <= 128) return heads(i8, std::integral_constant<int, 128>{});
    if (widest <= 192) return heads(i8, std::integral_constant<int, 192>{});
    return heads(i8, std::integral_constant<int, 256>{});
  };
  return int8 ? size(std::true_type{}) : size(std::false_type{});
}
struct CtasPerSm {
  template <bool kInt8, int DP, int kHeads> int operator()() const { return Shape<kInt8, DP, kHeads>::kCtasPerSm; }
};
struct TileTokens {
  template <bool kInt8, int DP, int kHeads> int operator()() const { return Shape<kInt8, DP, kHeads>::kTile; }
};
struct Launch {
  const PagedAttnParams& p;
  bool cluster;
  cudaStream_t s;
  template <bool kInt8, int DP, int kHeads> msd_status_t operator()() const { return launch_paged<kInt8, DP, kHeads>(p, cluster, s); }
};

}  // namespace

}  // namespace msd

extern "C" {

size_t msd_attn_decode_paged_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t Dv, int64_t ld) {
  size_t most = 0;                              // of the kernels that a size of the keys may choose
  for (int widest : {192, 256}) {
    msd::PagedPlan pl;
    if (!msd::plan_paged(B, Hq, Hkv, Dv, ld, msd::head_slots(Hkv < 1 ? 1 : Hq / Hkv, widest), 4, &pl)) return 0;
    if (pl.bytes > most) most = pl.bytes;
  }
  return most;
}

msd_status_t msd_attn_decode_paged(const void* q_bf16, int64_t q_ld, const msd_paged_cache_t* cache, const int32_t* block_table,
                                   int32_t max_blocks, const int32_t* seqlens, int32_t B, int32_t Hq, float softmax_scale, void* out_bf16,
                                   float* lse, float* weights, int64_t ld, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace msd;
  PagedAttnParams p;
  if (const msd_status_t st = paged_cache_view(cache, &p.c)) return st;
  if (B < 0 || max_blocks < 1 || Hq < 1 || Hq % cache->Hkv != 0 || (weights && ld < 1) || (weights && ld > 0x7FFFFFFF)) return MSD_ERR_BAD_SHAPE;
  if (q_ld < static_cast<int64_t>(Hq) * cache->D) return MSD_ERR_BAD_SHAPE;
  if (B == 0) return MSD_OK;
  const bool int8 = cache->type == MSD_CACHE_INT8;
  const int widest = cache->D > cache->Dv ? cache->D : cache->Dv, slots = head_slots(Hq / cache->Hkv, widest);
  PagedPlan pl;
  const int ctas_per_sm = with_shape(int8, widest, slots, CtasPerSm{});
  if (!plan_paged(B, Hq, cache->Hkv, cache->Dv, weights ? ld : 0, slots, ctas_per_sm, &pl)) return MSD_ERR_UNSUPPORTED;
  if (!q_bf16 || !block_table || !seqlens || !out_bf16 || !workspace) return MSD_ERR_NULL_POINTER;
  if (!aligned(q_bf16, 16) || q_ld % 8 != 0 || !aligned(out_bf16, 16) || !aligned(workspace, 1024) || !aligned(block_table, 4) ||
      !aligned(seqlens, 4) || !aligned(lse, 4) || !aligned(weights, 4))
    return MSD_ERR_BAD_ALIGNMENT;
  if (workspace_bytes < pl.bytes) return MSD_ERR_WORKSPACE_TOO_SMALL;
  // A query is read by all runs of its sequence and KV head; the first to end may write.  Rows of q that end behind the start of `out`
  // and begin before its end:
  const int64_t q_row = static_cast<int64_t>(Hq) * cache->D * 2, out_bytes = static_cast<int64_t>(B) * Hq * cache->Dv * 2;
  const __int128 q_end = static_cast<__int128>(reinterpret_cast<uintptr_t>(out_bf16)) - reinterpret_cast<uintptr_t>(q_bf16) - q_row, step = static_cast<__int128>(q_ld) * 2;
  const __int128 row = q_end < 0 ? 0 : q_end / step + 1;       // the first that ends behind the start of `out`
  if (row < B && row * step < q_end + q_row + out_bytes) return MSD_ERR_UNSUPPORTED;
  const int64_t page = cache->page_size, blocks = cache->num_blocks, most_rows = int64_t{1} << 36, most_scales = int64_t{1} << 34;
  if (!rows_within(p.c.k, blocks, page, most_rows) || !rows_within(p.c.v, blocks, page, most_rows) ||
      (int8 && !(rows_within(p.c.ks, blocks, page, most_scales) && rows_within(p.c.vs, blocks, page, most_scales))))
    return MSD_ERR_UNSUPPORTED;
  // (positions stay below 2^31 - the tokens of a tile, and tiles below 2^31, so that no sum of theirs wraps)
  p.cap = static_cast<int64_t>(max_blocks) * cache->page_size;
  if (p.cap > 0x7FFFF000) p.cap = 0x7FFFF000;
  const int tile = with_shape(int8, widest, slots, TileTokens{});
  const int64_t room = (p.cap + tile - 1) / tile * B;      // tiles; of the table alone: the schedule, and so the bits, do not depend on the weights
  if (room > 0x7FFFFFFF) return MSD_ERR_UNSUPPORTED;
  if (weights && p.cap > ld) p.cap = ld;
  p.k_block = static_cast<uint32_t>(p.c.k.block / 16);
  p.k_token = static_cast<uint32_t>(p.c.k.token / 16);
  p.v_block = static_cast<uint32_t>(p.c.v.block / 16);
  p.v_token = static_cast<uint32_t>(p.c.v.token / 16);
  p.ks_block = static_cast<uint32_t>(p.c.ks.block / 4);
  p.ks_token = static_cast<uint32_t>(p.c.ks.token / 4);
  p.vs_block = static_cast<uint32_t>(p.c.vs.block / 4);
  p.vs_token = static_cast<uint32_t>(p.c.vs.token / 4);
  p.status = device_status_ptr();
  if (!p.status) return MSD_ERR_CUDA;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.q = static_cast<const uint16_t*>(q_bf16);
  p.q_ld = q_ld;
  p.table = block_table;
  p.seqlens = seqlens;
  p.max_blocks = max_blocks;
  // Keys and values that L2 can hold a part of until the next step leave it before anything else does, or a part of them is never there
  // when it is asked for again.  (Measured on caches that the next call reads again; between a model's layers little of one is left, and either will do.)
  // 64/8 heads, 24 x 512-4096 tokens INT8 34.3 / 32.4 us without / with, 16/16 heads of 80, 48 x 0-1500 51 / 47;
  // of more than that nothing stays either way, and it costs 3 % (2 x 100000-131072 BF16 164 / 169 us).
  p.leave_l2 = static_cast<double>(p.cap) * B * cache->Hkv * (cache->D + cache->Dv) * (int8 ? 1 : 2) <= 512e6;
  p.B = B;
  p.Hq = Hq;
  p.G = Hq / cache->Hkv;
  p.groups = pl.groups;
  p.U = pl.U;
  // no more runs than tiles that the sequences have room for (their lengths are on the device)
  p.runs = room < pl.runs ? static_cast<int>(room) : pl.runs;
  // Few tiles: one kernel, in which the runs of a unit are a cluster.  It saves a launch and the second kernel's first loads, but has at most 16
  // runs; so a CTA has no more tiles than in the other form, or up to four of a single sequence (a second sequence costs more than a second
  // tile).  32/8 heads of 128 on the GPU, two kernels / one: BF16 1 x 1000 tokens 8.0 / 6.9 us, 1 x 4000 13.1 / 9.7, 4 x 128-256 with weights 7.8 /
  // 7.1, INT8 1 x 4000 with weights 11.9 / 10.4, 8 x 128-256 9.3 / 8.4; 16 x 32-64 with weights 6.9 / 7.5.  The call's host time goes from 6.4 to 4.2 us.
  // (`room` is the table's: with a table for more tokens, short sequences are read by two kernels as well.)
  bool cluster = false;
  if (slots == 8) {
    int runs = 1;
    const int most = ctas_per_sm == 1 ? kClusterCtas / 2 : kClusterCtas;        // (a cluster lies on the SMs of one GPC)
    while (runs < room && runs * 2 <= pl.runs && runs < most) runs *= 2;
    const int64_t tiles = (room + pl.runs - 1) / pl.runs;        // of a CTA in the other form
    cluster = room <= runs * (B == 1 ? kClusterTiles : (tiles < kClusterTiles ? tiles : kClusterTiles));
    if (cluster) p.runs = runs;
  }
  p.scale2 = softmax_scale * 1.4426950408889634f;
  p.out = static_cast<uint16_t*>(out_bf16);
  p.lse = lse;
  p.weights = weights;
  p.ld = ld;
  p.score_ld = ld;
  p.score_heads = pl.score_heads;
  p.slots = pl.slots;
  p.part = reinterpret_cast<float*>(ws + pl.part);
  p.part_ml = reinterpret_cast<float*>(ws + pl.ml);
  p.tail = reinterpret_cast<int4*>(ws + pl.tail);
  p.seq_runs = reinterpret_cast<int2*>(ws + pl.seq_runs);
  p.lse2 = reinterpret_cast<float*>(ws + pl.lse2);
  p.scores = reinterpret_cast<float*>(ws + pl.scores);
  p.part_rows = pl.part_rows;
  // as many CTAs for the weights as fill the machine a few times, none with less than a block of positions
  const int64_t most = (ld + kJoinThreads - 1) / kJoinThreads, fill = (4LL * sm_count() + static_cast<int64_t>(B) * cache->Hkv - 1) / (static_cast<int64_t>(B) * cache->Hkv);
  p.join_weight_ctas = static_cast<int>(most < fill ? (most < 1 ? 1 : most) : fill);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_shape(int8, widest, slots, Launch{p, cluster, s});
}

}  // extern "C"
