// Decode attention of one new token per sequence over a paged cache (BF16, or INT8 codes with one scale per token and KV head),
// with the attention weight of every cached token summed up on the way (msd_attn_decode_paged).
//
//   S_hj = scale q_h.k_j,  P = softmax(S),  out = P V,  weights_j += sum_h P_hj
//
// Bound: HBM.  A token of a KV head is 2 (D + Dv) bytes (BF16) for 2 G (D + Dv) multiply-adds of its G query heads.  An SM takes in
// 44 bytes a nanosecond, 23 a clock, and the warp-level MMAs of that (16 head slots, used or not) are a fifth of what the pipe does,
// so nothing here waits for the tensor cores, and what counts is that loads never stop.  Hence no roles and no hand-offs: each warp
// keeps a ring of token tiles of its own in flight (cp.async, a row's page looked up a tile ahead), multiplies a tile against the
// query fragments in its registers, keeps its own running maximum, sum and output, and meets the other warps of its CTA only
// when a sequence ends.
//
// Fragments (mma m16n8k16): heads are the 16 rows; the scores of 8 tokens are a C fragment, which is the A fragment of the product
// with v as it stands.  INT8 codes go from shared memory to registers as bytes and become BF16 pairs there (exact): a byte x is
// (128 + (x & 127)) - (128 + (x & 128)), two byte permutes, masks and one packed subtraction for a pair.
//
// Split over the length: the tiles of all sequences form one list, cut into equal runs; run i is walked by U = KV heads x head groups
// CTAs side by side, one per unit, so that CTAs that run together read neighbouring rows.  The grid is what is resident at once.
// A sequence inside one run is finished there; only the first and the last of a run can be cut, so a CTA leaves at most two
// partial results, whatever the lengths are, and a second kernel joins those and turns the scores into weights.
#include <cuda_bf16.h>

#include <cmath>

#include "paged.cuh"

namespace msd {

namespace {

constexpr int kPWarps = 4;
constexpr int kPThreads = 32 * kPWarps;
constexpr int kPRows = 16;                  // head slots of a CTA (MMA rows)
constexpr int kJoinThreads = 256;

struct PagedAttnParams {
  PagedCache c;
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
  // workspace
  float* part;                // [CTA][2][rows][Dv]: unnormalised outputs
  float* part_ml;             // [CTA][2][rows][2]: maximum (log2) and sum
  int2* tail;                 // [CTA] what the join does for it: {sequence cut at the end of its run or -1, last run of that sequence}
  int2* seq_runs;             // [B] {first, last run}
  float* lse2;                // [B, Hq] log2-sum of uncut sequences
  float* scores;              // [B, Hq, score_ld] log2 scores
  int part_rows;              // rows of a partial result: min(G, 16)
  int join_weight_ctas;       // CTAs of the join per (sequence, KV head)
  unsigned* status;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {       // zeros where there is nothing
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// bytes kLo and kHi of r (two's complement) as a BF16 pair
template <int kLo, int kHi>
__device__ __forceinline__ uint32_t int8_pair(uint32_t r) {
  const uint32_t t = __byte_perm(r, 0x43u, 0x4040 | kLo | (kHi << 8));        // each byte below 0x43: 128 + (x & 127), and the sign as bit 7
  const uint32_t low = t & 0xFF7FFF7Fu, sign = t & 0xFF80FF80u;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&low), *reinterpret_cast<const __nv_bfloat162*>(&sign));
  return *reinterpret_cast<const uint32_t*>(&d);
}

// DP: D and Dv rounded up to 64, 128 or 256.  A tile of a warp: 8 KB of keys and values where that is 16 or 32 tokens; three of them in
// flight and two CTAs an SM put 200 KB of loads under way, four times what the latency of a loaded memory asks for.
template <bool kInt8, int DP>
struct Shape {
  static constexpr int kEs = kInt8 ? 1 : 2;
  static constexpr int kTok = (DP == 64 || (kInt8 && DP == 128)) ? 32 : 16;
  static constexpr int kRow = DP * kEs;                         // bytes of a row in shared memory
  static constexpr int kHalf = kTok * kRow;                     // keys, then values
  static constexpr int kScale = kInt8 ? kTok * 4 : 0;           // then the scales of both
  static constexpr int kStage = 2 * kHalf + 2 * kScale;
  static constexpr int kStages = kInt8 ? (DP == 64 ? 4 : (DP == 256 ? 6 : 3)) : 3;
  static constexpr int kCtasPerSm = DP == 256 ? 1 : 2;
  static constexpr bool kQInSmem = DP == 256;                   // (64 registers of query fragments beside 128 of outputs are too many)
  static constexpr int kQRow = DP * 2 + 16;                     // bytes: rows 16 bytes apart in the banks
  static constexpr int kRing = kPWarps * kStages * kStage;
  static constexpr int kOut = kPRows * (DP + 4) * 4;            // where the warps' outputs meet
  static constexpr int kSmem = kRing + kOut + (kQInSmem ? kPRows * kQRow : 0);
  static constexpr int kTile = kPWarps * kTok;                  // tokens of a CTA's tile
  static_assert(kCtasPerSm * (kSmem + 2048) <= 228 * 1024, "the CTAs of an SM have to fit its shared memory");
};

// 16-byte chunk c of row r, so that the eight rows of a matrix lie in different banks
template <int kRow>
__device__ __forceinline__ uint32_t swz(int r, int c) {
  return r * kRow + ((c ^ (kRow >= 128 ? (r & 7) : ((r >> 1) & 3))) << 4);
}

__device__ __forceinline__ int seq_len(const PagedAttnParams& p, int b) {
  const int32_t n = p.seqlens[b];
  return static_cast<int>(min(static_cast<int64_t>(n < 0 ? 0 : n), p.cap));
}

template <bool kInt8, int DP>
__global__ void __launch_bounds__(kPThreads, (Shape<kInt8, DP>::kCtasPerSm))
attn_paged_kernel(const __grid_constant__ PagedAttnParams p) {
  using S = Shape<kInt8, DP>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int scan_buf[kPWarps];
  __shared__ int start_buf[2];
  __shared__ float ml[2][kPWarps][kPRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int unit = blockIdx.x % p.U, run = blockIdx.x / p.U;
  const int hk = unit / p.groups, h0 = (unit - hk * p.groups) * kPRows;        // first head of the group within the KV head
  const int nh = min(p.G - h0, kPRows);
  const int64_t head0 = static_cast<int64_t>(hk) * p.G + h0;

  pdl_wait_primary();
  pdl_launch_dependents();

  // ---- this CTA's run of tiles ----
  const int b_first = threadIdx.x;
  int total = 0, tiles_first = 0;
  for (int b = b_first; b < p.B; b += kPThreads) {
    const int32_t n = p.seqlens[b];
    const int L = seq_len(p, b);
    if (L != n && unit == 0 && run == 0) atomicMax(p.status, kStatusBadShape);
    const int t = (L + S::kTile - 1) / S::kTile;
    if (b == b_first) tiles_first = t;
    total += t;
    if (L == 0 && b % p.runs == run) {           // nothing to attend to
      for (int h = 0; h < nh; ++h) {
        const int64_t row = static_cast<int64_t>(b) * p.Hq + head0 + h;
        for (int d = 0; d < p.c.Dv; d += 8) *reinterpret_cast<uint4*>(p.out + row * p.c.Dv + d) = make_uint4(0, 0, 0, 0);
        if (p.lse) p.lse[row] = -INFINITY;
      }
    }
  }
  auto block_scan = [&](int v, int* sum) {       // inclusive, over the threads of the block
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) scan_buf[warp] = x;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kPWarps; ++w) {
      if (w < warp) x += scan_buf[w];
      all += scan_buf[w];
    }
    *sum = all;
    return x;
  };
  int T;
  block_scan(total, &T);
  if (threadIdx.x == 0) p.tail[blockIdx.x] = make_int2(-1, 0);
  const int runs = min(p.runs, T);                // (no empty runs)
  if (run >= runs) return;
  auto run_start = [&](int r) { return static_cast<int>(static_cast<int64_t>(r) * T / runs); };
  const int first = run_start(run), end = run_start(run + 1);
  for (int base = 0, carry = 0; base < p.B && carry <= first; base += kPThreads) {
    const int b = base + threadIdx.x;
    const int t = base == 0 ? tiles_first : (b < p.B ? (seq_len(p, b) + S::kTile - 1) / S::kTile : 0);
    int sum;
    const int incl = carry + block_scan(t, &sum);
    if (first >= incl - t && first < incl) { start_buf[0] = b; start_buf[1] = first - (incl - t); }
    carry += sum;
  }
  __syncthreads();

  // A walk over the tiles of the run, one for the loads and one for the arithmetic.
  struct Walk {
    int b, tile, tiles, L, left;          // sequence, tile of it, tiles of it, its length, tiles left in the run
  };
  Walk ld;
  ld.b = start_buf[0];
  ld.tile = start_buf[1];
  ld.L = seq_len(p, ld.b);
  ld.tiles = (ld.L + S::kTile - 1) / S::kTile;
  ld.left = end - first;
  Walk cur = ld;
  auto advance = [&](Walk& w) {
    --w.left;
    if (++w.tile == w.tiles && w.left > 0) {
      do {
        w.L = seq_len(p, ++w.b);
      } while (w.L == 0);
      w.tile = 0;
      w.tiles = (w.L + S::kTile - 1) / S::kTile;
    }
  };

  // ---- loads ----
  uint8_t* ring = smem + warp * (S::kStages * S::kStage);
  const uint32_t ring_u = smem_u32(ring);
  const uint8_t* kbase = p.c.k.base + hk * p.c.k.head;
  const uint8_t* vbase = p.c.v.base + hk * p.c.v.head;
  constexpr int kChunks = S::kRow / 16;                 // 16-byte chunks of a row
  constexpr int kRowsPer = 32 / kChunks;                // rows that one instruction of the warp brings
  const int k_chunks = p.c.D * S::kEs / 16, v_chunks = p.c.Dv * S::kEs / 16;
  const int my_chunk = lane % kChunks, my_row = lane / kChunks;
  const int tok_lane = lane & (S::kTok - 1);
  // the block of this lane's token of the tile that `ld` stands on, asked for a tile ahead
  auto look_up = [&](const Walk& w) -> int {
    const int pos = w.tile * S::kTile + warp * S::kTok + tok_lane;
    if (w.left <= 0 || pos >= w.L) return -1;
    return p.table[static_cast<int64_t>(w.b) * p.max_blocks + div_by(pos, p.c.page)];
  };
  int blk = look_up(ld);
  auto issue = [&](int stage) {
    if (ld.left > 0) {
      const int pos = ld.tile * S::kTile + warp * S::kTok + tok_lane;
      bool there = pos < ld.L;
      if (there && static_cast<uint32_t>(blk) >= static_cast<uint64_t>(p.c.num_blocks)) {
        atomicMax(p.status, kStatusBadShape);
        there = false;
      }
      const uint32_t slot = pos - div_by(pos, p.c.page) * p.c.page.d;
      const int64_t ko = there ? row_offset(p.c.k, blk, slot) : -1, vo = there ? row_offset(p.c.v, blk, slot) : -1;
      const uint32_t dst = ring_u + stage * S::kStage;
#pragma unroll
      for (int i = 0; i < S::kTok / kRowsPer; ++i) {
        const int r = i * kRowsPer + my_row;
        const int64_t o = __shfl_sync(0xffffffffu, ko, r);
        const bool ok = o >= 0 && my_chunk < k_chunks;
        cp16(dst + swz<S::kRow>(r, my_chunk), kbase + (ok ? o + my_chunk * 16 : 0), ok);
      }
#pragma unroll
      for (int i = 0; i < S::kTok / kRowsPer; ++i) {
        const int r = i * kRowsPer + my_row;
        const int64_t o = __shfl_sync(0xffffffffu, vo, r);
        const bool ok = o >= 0 && my_chunk < v_chunks;
        cp16(dst + S::kHalf + swz<S::kRow>(r, my_chunk), vbase + (ok ? o + my_chunk * 16 : 0), ok);
      }
      if constexpr (kInt8) {
        const uint32_t sc = dst + 2 * S::kHalf + tok_lane * 4;
        const int64_t kso = there ? row_offset(p.c.ks, blk, slot) + hk * p.c.ks.head : 0;
        const int64_t vso = there ? row_offset(p.c.vs, blk, slot) + hk * p.c.vs.head : 0;
        if (S::kTok == 32 || lane < 16) cp4(sc, p.c.ks.base + kso, there);
        if (S::kTok == 32 || lane >= 16) cp4(sc + S::kScale, p.c.vs.base + vso, there);
      }
      advance(ld);
      blk = look_up(ld);
    }
    cp_commit();
  };
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) issue(s);

  // ---- the arithmetic ----
  const int row = lane >> 2, quad = lane & 3;           // rows `row` and `row` + 8 of the fragments
  uint8_t* sm_q = smem + S::kRing + S::kOut;
  float* sm_o = reinterpret_cast<float*>(smem + S::kRing);
  constexpr int kSteps = DP / 16;
  uint32_t qf[S::kQInSmem ? 1 : kSteps][4];
  float o[DP / 8][4];
  float m0, m1, l0, l1;
  const int k_steps = (p.c.D + 15) / 16;

  auto load_q = [&]() {
    const uint16_t* q = p.q + static_cast<int64_t>(cur.b) * p.q_ld + head0 * p.c.D;
    if constexpr (S::kQInSmem) {
      for (int i = threadIdx.x; i < kPRows * (DP / 8); i += kPThreads) {
        const int r = i / (DP / 8), c = i % (DP / 8);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < nh && c * 8 < p.c.D) v = *reinterpret_cast<const uint4*>(q + r * p.c.D + c * 8);
        *reinterpret_cast<uint4*>(sm_q + r * S::kQRow + c * 16) = v;
      }
      __syncthreads();
    } else {
      // INT8: of 16 values of d a thread's bytes are 4 quad ... 4 quad + 3, so the query is taken in that order too
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = row + (j & 1) * 8;
          const int d = s * 16 + (kInt8 ? 4 * quad + (j >> 1) * 2 : 2 * quad + (j >> 1) * 8);
          qf[s][j] = (r < nh && d < p.c.D) ? *reinterpret_cast<const uint32_t*>(q + r * p.c.D + d) : 0u;
        }
      }
    }
  };
  auto q_fragment = [&](int s, uint32_t (&a)[4]) {
    if constexpr (!S::kQInSmem) {
#pragma unroll
      for (int j = 0; j < 4; ++j) a[j] = qf[s][j];
    } else if constexpr (kInt8) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint2 v = *reinterpret_cast<const uint2*>(sm_q + (row + j * 8) * S::kQRow + s * 32 + quad * 8);
        a[j] = v.x;
        a[j + 2] = v.y;
      }
    } else {
      ldsm4(a, smem_u32(sm_q) + (lane & 15) * S::kQRow + s * 32 + (lane >> 4) * 16);
    }
  };

  int it = 0;
  while (cur.left > 0) {
    // a segment: the tiles of one sequence that are in this run
    const int seg_first = cur.tile;
    const int seg = min(cur.tiles - cur.tile, cur.left);
    const int b = cur.b, L = cur.L;
    load_q();
    m0 = m1 = -INFINITY;
    l0 = l1 = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;

    for (int t = 0; t < seg; ++t, ++it) {
      const int stage = it % S::kStages;
      cp_wait<S::kStages - 2>();
      __syncwarp();
      issue((it + S::kStages - 1) % S::kStages);        // the stage that the last tile left
      const int pos0 = cur.tile * S::kTile + warp * S::kTok;
      advance(cur);
      if (pos0 >= L) continue;                          // (uniform in the warp)
      const uint32_t sk = ring_u + stage * S::kStage, sv = sk + S::kHalf;
      const float* scales = reinterpret_cast<const float*>(ring + stage * S::kStage + 2 * S::kHalf);

      // scores
      float s[S::kTok / 8][4];
#pragma unroll
      for (int n = 0; n < S::kTok / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
      if constexpr (kInt8) {
#pragma unroll
        for (int c4 = 0; c4 < DP / 64; ++c4) {
          if (c4 * 4 < k_steps) {
            uint32_t a[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q_fragment(c4 * 4 + i, a[i]);
#pragma unroll
            for (int n = 0; n < S::kTok / 8; ++n) {
              uint32_t r[4];
              ldsm4(r, sk + swz<S::kRow>(n * 8 + (lane & 7), c4 * 4 + (lane >> 3)));
#pragma unroll
              for (int i = 0; i < 4; ++i) mma_bf16(s[n], a[i], int8_pair<0, 1>(r[i]), int8_pair<2, 3>(r[i]));
            }
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
          if (c < k_steps) {
            uint32_t a[4];
            q_fragment(c, a);
#pragma unroll
            for (int n = 0; n < S::kTok / 8; n += 2) {
              uint32_t r[4];
              ldsm4(r, sk + swz<S::kRow>(n * 8 + ((lane >> 4) << 3) + (lane & 7), 2 * c + ((lane >> 3) & 1)));
              mma_bf16(s[n], a, r[0], r[1]);
              mma_bf16(s[n + 1], a, r[2], r[3]);
            }
          }
        }
      }

      // softmax
      float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
      for (int n = 0; n < S::kTok / 8; ++n) {
        float f0 = p.scale2, f1 = p.scale2;
        if constexpr (kInt8) {
          const float2 ks = *reinterpret_cast<const float2*>(scales + n * 8 + 2 * quad);
          f0 *= ks.x;
          f1 *= ks.y;
        }
        s[n][0] *= f0;
        s[n][1] *= f1;
        s[n][2] *= f0;
        s[n][3] *= f1;
      }
      if (pos0 + S::kTok > L) {
#pragma unroll
        for (int n = 0; n < S::kTok / 8; ++n) {
          const int pos = pos0 + n * 8 + 2 * quad;
          if (pos >= L) s[n][0] = s[n][2] = -INFINITY;
          if (pos + 1 >= L) s[n][1] = s[n][3] = -INFINITY;
        }
      }
      if (p.weights) {
        float* dst = p.scores + (static_cast<int64_t>(b) * p.Hq + head0 + row) * p.score_ld + pos0 + 2 * quad;
#pragma unroll
        for (int n = 0; n < S::kTok / 8; ++n) {
          if (pos0 + n * 8 + 2 * quad < L) {
            if (row < nh) *reinterpret_cast<float2*>(dst + n * 8) = make_float2(s[n][0], s[n][1]);
            if (row + 8 < nh) *reinterpret_cast<float2*>(dst + 8 * p.score_ld + n * 8) = make_float2(s[n][2], s[n][3]);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < S::kTok / 8; ++n) {
        mx0 = fmaxf(mx0, fmaxf(s[n][0], s[n][1]));
        mx1 = fmaxf(mx1, fmaxf(s[n][2], s[n][3]));
      }
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, d));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, d));
      }
      mx0 = fmaxf(mx0, m0);
      mx1 = fmaxf(mx1, m1);
      if (__any_sync(0xffffffffu, mx0 != m0 || mx1 != m1)) {
        const float r0 = mx0 == -INFINITY ? 1.0f : ex2(m0 - mx0), r1 = mx1 == -INFINITY ? 1.0f : ex2(m1 - mx1);
        m0 = mx0;
        m1 = mx1;
        l0 *= r0;
        l1 *= r1;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
          o[i][0] *= r0;
          o[i][1] *= r0;
          o[i][2] *= r1;
          o[i][3] *= r1;
        }
      }
      const float e0 = m0 == -INFINITY ? 0.0f : m0, e1 = m1 == -INFINITY ? 0.0f : m1;
#pragma unroll
      for (int n = 0; n < S::kTok / 8; ++n) {
        s[n][0] = ex2(s[n][0] - e0);
        s[n][1] = ex2(s[n][1] - e0);
        s[n][2] = ex2(s[n][2] - e1);
        s[n][3] = ex2(s[n][3] - e1);
        l0 += s[n][0] + s[n][1];
        l1 += s[n][2] + s[n][3];
      }

      // product with v, 16 tokens at a time
#pragma unroll
      for (int g = 0; g < S::kTok / 16; ++g) {
        if constexpr (kInt8) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 vs = *reinterpret_cast<const float2*>(scales + S::kTok + (2 * g + j) * 8 + 2 * quad);
            s[2 * g + j][0] *= vs.x;
            s[2 * g + j][1] *= vs.y;
            s[2 * g + j][2] *= vs.x;
            s[2 * g + j][3] *= vs.y;
          }
        }
        const uint32_t a[4] = {pack_bf16(s[2 * g][0], s[2 * g][1]), pack_bf16(s[2 * g][2], s[2 * g][3]),
                               pack_bf16(s[2 * g + 1][0], s[2 * g + 1][1]), pack_bf16(s[2 * g + 1][2], s[2 * g + 1][3])};
#pragma unroll
        for (int c = 0; c < kChunks; c += 2) {
          if (c < v_chunks) {
            uint32_t r[4];
            ldsm4_t(r, sv + swz<S::kRow>(g * 16 + (lane & 15), c + (lane >> 4)));
            if constexpr (kInt8) {      // a register holds two tokens of an even and the next odd value of d
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                mma_bf16(o[2 * (c + j)], a, int8_pair<0, 2>(r[2 * j]), int8_pair<0, 2>(r[2 * j + 1]));
                mma_bf16(o[2 * (c + j) + 1], a, int8_pair<1, 3>(r[2 * j]), int8_pair<1, 3>(r[2 * j + 1]));
              }
            } else {
              mma_bf16(o[c], a, r[0], r[1]);
              mma_bf16(o[c + 1], a, r[2], r[3]);
            }
          }
        }
      }
    }

    // ---- the segment's end: the warps meet ----
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, d);
      l1 += __shfl_xor_sync(0xffffffffu, l1, d);
    }
    if (quad == 0) {
      ml[0][warp][row] = m0;
      ml[0][warp][row + 8] = m1;
      ml[1][warp][row] = l0;
      ml[1][warp][row + 8] = l1;
    }
    __syncthreads();
    auto joined = [&](int r, float* m, float* l) {
      float mm = ml[0][0][r];
#pragma unroll
      for (int w = 1; w < kPWarps; ++w) mm = fmaxf(mm, ml[0][w][r]);
      float ll = 0.0f;
#pragma unroll
      for (int w = 0; w < kPWarps; ++w) ll += ml[1][w][r] * (ml[0][w][r] == -INFINITY ? 0.0f : ex2(ml[0][w][r] - mm));
      *m = mm;
      *l = ll;
    };
    float M0, M1, L0, L1;
    joined(row, &M0, &L0);
    joined(row + 8, &M1, &L1);
    const float f0 = m0 == -INFINITY ? 0.0f : ex2(m0 - M0), f1 = m1 == -INFINITY ? 0.0f : ex2(m1 - M1);
    constexpr int kORow = DP + 4;
    for (int w = 0; w < kPWarps; ++w) {          // one after the other: the order of the sums is fixed
      if (w == warp) {
#pragma unroll
        for (int i = 0; i < DP / 8; i += 2) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float f = j ? f1 : f0;
            const int r = row + 8 * j;
            if (r < nh) {
              float x[4] = {o[i][2 * j] * f, o[i][2 * j + 1] * f, o[i + 1][2 * j] * f, o[i + 1][2 * j + 1] * f};
              if constexpr (kInt8) {             // columns 2 quad, 2 quad + 1 of a pair of fragments are four values in a row
                float4* dst = reinterpret_cast<float4*>(sm_o + r * kORow + i * 8 + 4 * quad);
                float4 v = make_float4(x[0], x[2], x[1], x[3]);
                if (w > 0) { const float4 y = *dst; v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w; }
                *dst = v;
              } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  float2* dst = reinterpret_cast<float2*>(sm_o + r * kORow + (i + k) * 8 + 2 * quad);
                  float2 v = make_float2(x[2 * k], x[2 * k + 1]);
                  if (w > 0) { const float2 y = *dst; v.x += y.x; v.y += y.y; }
                  *dst = v;
                }
              }
            }
          }
        }
      }
      __syncthreads();
    }
    const bool from_start = seg_first == 0, to_end = seg_first + seg == (L + S::kTile - 1) / S::kTile;
    const int Dv = p.c.Dv, vecs = Dv / 4;
    if (from_start && unit == 0 && threadIdx.x == 0) {
      const int64_t at = first + (static_cast<int64_t>(end - first) - cur.left - seg);      // the sequence's first tile in the list
      const int64_t last = at + (L + S::kTile - 1) / S::kTile - 1;
      p.seq_runs[b] = make_int2(run, static_cast<int>(((last + 1) * runs - 1) / T));
    }
    if (from_start && to_end) {
      for (int i = threadIdx.x; i < nh * vecs; i += kPThreads) {
        const int r = i / vecs, d = (i - r * vecs) * 4;
        float m, l;
        joined(r, &m, &l);
        const float inv = 1.0f / l;
        const float4 v = *reinterpret_cast<const float4*>(sm_o + r * kORow + d);
        const uint2 w = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
        const int64_t out_row = static_cast<int64_t>(b) * p.Hq + head0 + r;
        *reinterpret_cast<uint2*>(p.out + out_row * Dv + d) = w;
        if (d == 0) {
          const float lg = m + log2f(l);
          if (p.lse) p.lse[out_row] = lg * 0.6931471805599453f;
          if (p.weights) p.lse2[out_row] = lg;
        }
      }
    } else {
      const int64_t slot = static_cast<int64_t>(blockIdx.x) * 2 + (from_start ? 1 : 0);
      for (int i = threadIdx.x; i < nh * vecs; i += kPThreads) {
        const int r = i / vecs, d = (i - r * vecs) * 4;
        *reinterpret_cast<float4*>(p.part + (slot * p.part_rows + r) * Dv + d) = *reinterpret_cast<const float4*>(sm_o + r * kORow + d);
        if (d == 0) {
          float m, l;
          joined(r, &m, &l);
          *reinterpret_cast<float2*>(p.part_ml + (slot * p.part_rows + r) * 2) = make_float2(m, l);
        }
      }
      if (from_start && threadIdx.x == 0) {
        const int64_t last = static_cast<int64_t>(end) + (L + S::kTile - 1) / S::kTile - seg - 1;
        p.tail[blockIdx.x] = make_int2(b, static_cast<int>(((last + 1) * runs - 1) / T));
      }
    }
    __syncthreads();
  }
  cp_wait<0>();
}

// Joins the partial results of cut sequences (CTAs [0, runs x U): the one where the sequence begins), and adds the attention weights
// (the other CTAs: (sequence, KV head) x share of the positions) from the scores that the first kernel left.
__global__ void __launch_bounds__(kJoinThreads)
attn_paged_join_kernel(const __grid_constant__ PagedAttnParams p) {
  __shared__ float f[kPRows * 2];
  __shared__ float4 sums[kJoinThreads];
  extern __shared__ float lse2_sm[];             // [G]
  pdl_wait_primary();
  pdl_launch_dependents();
  const int join_ctas = p.runs * p.U;
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) < join_ctas) {
    const int unit = blockIdx.x % p.U, run = blockIdx.x / p.U;
    const int2 tail = p.tail[blockIdx.x];
    if (tail.x < 0) return;
    const int hk = unit / p.groups, h0 = (unit - hk * p.groups) * kPRows, nh = min(p.G - h0, kPRows);
    const int n = tail.y - run + 1;              // pieces: slot 1 of this CTA, slot 0 of the runs after it
    auto slot = [&](int i) { return i == 0 ? static_cast<int64_t>(blockIdx.x) * 2 + 1 : (static_cast<int64_t>(run + i) * p.U + unit) * 2; };
    for (int r = tid >> 5; r < nh; r += kJoinThreads / 32) {       // a warp for each row's maximum and sum
      float m = -INFINITY, l = 0.0f;
      for (int i = tid & 31; i < n; i += 32) {
        const float2 x = *reinterpret_cast<const float2*>(p.part_ml + (slot(i) * p.part_rows + r) * 2);
        const float mn = fmaxf(m, x.x);
        if (mn != -INFINITY) l = l * ex2(m - mn) + x.y * ex2(x.x - mn);
        m = mn;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, d), ol = __shfl_xor_sync(0xffffffffu, l, d);
        const float mn = fmaxf(m, om);
        if (mn != -INFINITY) l = l * ex2(m - mn) + ol * ex2(om - mn);
        m = mn;
      }
      if ((tid & 31) == 0) {
        f[r] = m == -INFINITY ? 0.0f : m;
        f[kPRows + r] = 1.0f / l;
        if (p.lse) p.lse[static_cast<int64_t>(tail.x) * p.Hq + hk * p.G + h0 + r] = (m + log2f(l)) * 0.6931471805599453f;
      }
    }
    __syncthreads();
    const int vecs = p.c.Dv / 4, items = nh * vecs;
    const int share = items >= kJoinThreads ? 1 : kJoinThreads / items;          // threads that split an item's pieces
    for (int base = 0; base < items; base += kJoinThreads / share) {
      const int item = base + (tid / share), part = tid % share;
      const bool on = tid / share < kJoinThreads / share && item < items;
      float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (on) {
        const int r = item / vecs, d = (item - r * vecs) * 4;
#pragma unroll 4
        for (int i = part; i < n; i += share) {
          const int64_t s = slot(i) * p.part_rows + r;
          const float w = ex2(p.part_ml[s * 2] - f[r]);
          const float4 x = *reinterpret_cast<const float4*>(p.part + s * p.c.Dv + d);
          acc.x = fmaf(x.x, w, acc.x);
          acc.y = fmaf(x.y, w, acc.y);
          acc.z = fmaf(x.z, w, acc.z);
          acc.w = fmaf(x.w, w, acc.w);
        }
      }
      sums[tid] = acc;
      __syncthreads();
      if (on && part == 0) {
        for (int i = 1; i < share; ++i) {
          const float4 x = sums[tid + i];
          acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
        }
        const int r = item / vecs, d = (item - r * vecs) * 4;
        const float inv = f[kPRows + r];
        *reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(tail.x) * p.Hq + hk * p.G + h0 + r) * p.c.Dv + d) =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      }
      __syncthreads();
    }
    return;
  }

  const int w = blockIdx.x - join_ctas, share = w % p.join_weight_ctas, bk = w / p.join_weight_ctas;
  const int b = bk / p.c.Hkv, hk = bk - b * p.c.Hkv;
  const int L = seq_len(p, b);
  if (L == 0 || static_cast<int64_t>(share) * kJoinThreads >= L) return;
  const int2 span = p.seq_runs[b];
  for (int g = tid >> 5; g < p.G; g += kJoinThreads / 32) {
    float lg;
    if (span.x == span.y) {
      lg = p.lse2[static_cast<int64_t>(b) * p.Hq + hk * p.G + g];
    } else {
      const int unit = hk * p.groups + g / kPRows, r = g % kPRows;
      float m = -INFINITY, l = 0.0f;
      for (int i = tid & 31; i <= span.y - span.x; i += 32) {
        const int64_t slot = (static_cast<int64_t>(span.x + i) * p.U + unit) * 2 + (i == 0 ? 1 : 0);
        const float2 x = *reinterpret_cast<const float2*>(p.part_ml + (slot * p.part_rows + r) * 2);
        const float mn = fmaxf(m, x.x);
        if (mn != -INFINITY) l = l * ex2(m - mn) + x.y * ex2(x.x - mn);
        m = mn;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, d), ol = __shfl_xor_sync(0xffffffffu, l, d);
        const float mn = fmaxf(m, om);
        if (mn != -INFINITY) l = l * ex2(m - mn) + ol * ex2(om - mn);
        m = mn;
      }
      lg = m + log2f(l);
    }
    if ((tid & 31) == 0) lse2_sm[g] = lg;
  }
  __syncthreads();
  const float* s = p.scores + (static_cast<int64_t>(b) * p.Hq + static_cast<int64_t>(hk) * p.G) * p.score_ld;
  float* out = p.weights + (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.ld;
  for (int64_t j = static_cast<int64_t>(share) * kJoinThreads + tid; j < L; j += static_cast<int64_t>(p.join_weight_ctas) * kJoinThreads) {
    float acc = 0.0f;
#pragma unroll 4
    for (int g = 0; g < p.G; ++g) acc += ex2(s[g * p.score_ld + j] - lse2_sm[g]);
    out[j] += acc;
  }
}

struct PagedPlan {
  int groups, U, runs, part_rows;
  int64_t score_ld;
  size_t part, ml, tail, seq_runs, lse2, scores, bytes;     // offsets into the workspace
};

// (ctas_per_sm: 2 where the head dimension is not known; the workspace has room for that)
bool plan_paged(int B, int Hq, int Hkv, int Dv, int64_t ld, int ctas_per_sm, PagedPlan* pl) {
  if (B < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hq > 8192 || B > (1 << 20) || Dv < 1 || Dv > 256 || ld < 0 || ld > 0x7FFFFFFF) return false;
  const int G = Hq / Hkv;
  pl->groups = (G + kPRows - 1) / kPRows;
  pl->U = Hkv * pl->groups;
  pl->runs = sm_count() * ctas_per_sm / pl->U;
  if (pl->runs < 1) pl->runs = 1;
  pl->part_rows = G < kPRows ? G : kPRows;
  pl->score_ld = (ld + 3) / 4 * 4;
  const size_t ctas = static_cast<size_t>(pl->runs) * pl->U;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = round_up(at + bytes, 256);
    return o;
  };
  pl->part = take(ctas * 2 * pl->part_rows * Dv * 4);
  pl->ml = take(ctas * 2 * pl->part_rows * 8);
  pl->tail = take(ctas * sizeof(int2));
  pl->seq_runs = take(static_cast<size_t>(B) * sizeof(int2));
  pl->lse2 = take(static_cast<size_t>(B) * Hq * 4);
  pl->scores = take(static_cast<size_t>(B) * Hq * pl->score_ld * 4);
  pl->bytes = round_up(at, 1024);
  return true;
}

template <bool kInt8, int DP>
msd_status_t launch_paged(const PagedAttnParams& p, cudaStream_t s) {
  using Sh = Shape<kInt8, DP>;
  auto kernel = attn_paged_kernel<kInt8, DP>;
  static DeviceOnce once;
  if (!once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem) == cudaSuccess; })) return MSD_ERR_CUDA;
  const bool pdl = option(OPT_NO_PDL) != 1;
  if (launch_pdl(kernel, dim3(p.runs * p.U), dim3(kPThreads), Sh::kSmem, s, pdl, p) != cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }
  const unsigned weight_ctas = p.weights ? static_cast<unsigned>(p.B) * p.c.Hkv * p.join_weight_ctas : 0;
  if (launch_pdl(attn_paged_join_kernel, dim3(p.runs * p.U + weight_ctas), dim3(kJoinThreads), p.weights ? p.G * sizeof(float) : 0, s, pdl, p) !=
      cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }
  return MSD_OK;
}

}  // namespace

}  // namespace msd

extern "C" {

size_t msd_attn_decode_paged_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t Dv, int64_t ld) {
  msd::PagedPlan pl;
  return msd::plan_paged(B, Hq, Hkv, Dv, ld, 2, &pl) ? pl.bytes : 0;
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
  const int widest = cache->D > cache->Dv ? cache->D : cache->Dv, dp = widest <= 64 ? 64 : (widest <= 128 ? 128 : 256);
  PagedPlan pl;
  if (!plan_paged(B, Hq, cache->Hkv, cache->Dv, weights ? ld : 0, dp == 256 ? 1 : 2, &pl)) return MSD_ERR_UNSUPPORTED;
  if (!q_bf16 || !block_table || !seqlens || !out_bf16 || !workspace) return MSD_ERR_NULL_POINTER;
  if (!aligned(q_bf16, 16) || q_ld % 8 != 0 || !aligned(out_bf16, 16) || !aligned(workspace, 1024) || !aligned(block_table, 4) ||
      !aligned(seqlens, 4) || !aligned(lse, 4) || !aligned(weights, 4))
    return MSD_ERR_BAD_ALIGNMENT;
  if (workspace_bytes < pl.bytes) return MSD_ERR_WORKSPACE_TOO_SMALL;
  p.status = device_status_ptr();
  if (!p.status) return MSD_ERR_CUDA;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.q = static_cast<const uint16_t*>(q_bf16);
  p.q_ld = q_ld;
  p.table = block_table;
  p.seqlens = seqlens;
  p.max_blocks = max_blocks;
  // (positions stay below 2^31 - the tokens of a tile, so that no sum of theirs wraps)
  p.cap = static_cast<int64_t>(max_blocks) * cache->page_size;
  if (weights && p.cap > ld) p.cap = ld;
  if (p.cap > 0x7FFFF000) p.cap = 0x7FFFF000;
  p.B = B;
  p.Hq = Hq;
  p.G = Hq / cache->Hkv;
  p.groups = pl.groups;
  p.U = pl.U;
  p.runs = pl.runs;
  p.scale2 = softmax_scale * 1.4426950408889634f;
  p.out = static_cast<uint16_t*>(out_bf16);
  p.lse = lse;
  p.weights = weights;
  p.ld = ld;
  p.score_ld = pl.score_ld;
  p.part = reinterpret_cast<float*>(ws + pl.part);
  p.part_ml = reinterpret_cast<float*>(ws + pl.ml);
  p.tail = reinterpret_cast<int2*>(ws + pl.tail);
  p.seq_runs = reinterpret_cast<int2*>(ws + pl.seq_runs);
  p.lse2 = reinterpret_cast<float*>(ws + pl.lse2);
  p.scores = reinterpret_cast<float*>(ws + pl.scores);
  p.part_rows = pl.part_rows;
  // as many CTAs for the weights as fill the machine a few times, none with less than a block of positions
  const int64_t most = (ld + kJoinThreads - 1) / kJoinThreads, fill = (8LL * sm_count() + static_cast<int64_t>(B) * cache->Hkv - 1) / (static_cast<int64_t>(B) * cache->Hkv);
  p.join_weight_ctas = static_cast<int>(most < fill ? (most < 1 ? 1 : most) : fill);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (int8) return dp == 64 ? launch_paged<true, 64>(p, s) : (dp == 128 ? launch_paged<true, 128>(p, s) : launch_paged<true, 256>(p, s));
  return dp == 64 ? launch_paged<false, 64>(p, s) : (dp == 128 ? launch_paged<false, 128>(p, s) : launch_paged<false, 256>(p, s));
}

}  // extern "C"
