// A paged cache that is written (msd_kv_append_paged) and shortened (msd_kv_evict_paged).
#include <cuda_bf16.h>

#include "paged.cuh"
#include "quant.cuh"

namespace msd {

namespace {

__device__ __forceinline__ unsigned lanes_below(int lane) { return (1u << lane) - 1u; }

// ---------------------------------------------------------------------------------------------------------------------------
// Append.  Bound: HBM for prompts, a chain of latencies for one token a sequence.  A warp takes one new row and some of its KV heads:
// lanes 0-15 the key, lanes 16-31 the value (16 bytes a lane, twice where D > 128), so the largest element of a row is four
// shuffles away.  The rows are asked for before the warp looks for the sequence and the page they go to.  14480 rows of 8 heads of 128: BF16
// 22 us (5.4 TB/s), INT8 25.3 (3.6 TB/s; the arithmetic issues 60 % of the time); 64 rows INT8 2.6 us.
// ---------------------------------------------------------------------------------------------------------------------------
constexpr int kAppendThreads = 128;

struct AppendParams {
  PagedCache c;
  const uint16_t *k_new, *v_new;
  int64_t n_rows, k_ld, v_ld;
  const int32_t *table, *seqlens, *cu;
  int64_t cap;
  int max_blocks, B;
  int heads, head_groups;       // KV heads a warp takes, groups of them
  int row_ctas;                 // CTAs that take rows
  float* weights;
  int64_t ld;
  unsigned* status;
};

// The sequence that row n belongs to: cu[b] <= n < cu[b + 1], or -1 for rows before the first or behind the last one.  32 probes a step.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int64_t n, int lane) {
  int lo = 0, hi = B + 1;                       // cu[i] <= n for i < lo, cu[i] > n for i >= hi
  while (lo < hi) {
    const int span = hi - lo, step = (span + 31) / 32;
    const int i = lo + (lane + 1) * step - 1;   // the last of this lane's share
    const bool below = i < hi && cu[i] <= n;
    const int full = __popc(__ballot_sync(0xffffffffu, below));       // shares that end at or before n
    const int nlo = lo + full * step;
    hi = min(hi, nlo + step - 1);
    lo = min(nlo, hi);
  }
  return lo >= 1 && lo <= B ? lo - 1 : -1;
}

// m / 127 as a true division gives it: an estimate, corrected with its remainder twice, where no remainder underflows (Markstein's
// theorem: from a neighbour of the quotient and the rounded reciprocal, the correction with an exact remainder is the rounded quotient;
// P. Markstein, IBM J. Res. Dev. 34, 1990).
__device__ __forceinline__ float by_127(float m) {
  constexpr float kY = 1.0f / 127.0f;
  float q = m * kY;
  q = __fmaf_rn(__fmaf_rn(-127.0f, q, m), kY, q);
  return __fmaf_rn(__fmaf_rn(-127.0f, q, m), kY, q);
}

// 8 BF16 values -> 8 codes rne(fl(x / s)), two values an instruction and without a branch (rows are full of short integers over a short
// integer, whose quotients are ties or next to them).  s is fl(m / 127), m the row's largest value, inv about 1 / s.  The estimate x inv,
// corrected once with its exact remainder, is the quotient up to its last place.  Whether that is enough to round every one as its IEEE quotient rounds
// depends on the significands of x and m (seven bits each) and the difference of their exponents alone, so the test takes them all.  Adding
// 1.5 * 2^23 rounds half-to-even and leaves the code in the low byte.  (The largest quotient is 127 up to a unit: nothing to clamp.)
__device__ __forceinline__ uint2 codes_of(const uint4& v, float s, float inv) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  constexpr float kMagic = 12582912.0f;
  const uint64_t magic2 = pack_f32x2(kMagic, kMagic), inv2 = pack_f32x2(inv, inv), ns2 = pack_f32x2(-s, -s), zero2 = pack_f32x2(0.0f, 0.0f);
  uint32_t c[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t x = pack_f32x2(bf16lo(w[e]), bf16hi(w[e]));
    const uint64_t q = fma_f32x2(x, inv2, zero2);
    const float2 r = unpack_f32x2(add_f32x2(fma_f32x2(fma_f32x2(ns2, q, x), inv2, q), magic2));
    c[2 * e] = __float_as_uint(r.x);
    c[2 * e + 1] = __float_as_uint(r.y);
  }
  return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
}
// The same for a row whose largest value is tiny or huge, by true divisions, or no finite number: then the scale tells of it and the codes are 0.
__device__ __noinline__ uint2 codes_by_division(uint4 v, float s) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  unsigned long long out = 0;
#pragma unroll 1
  for (int e = 0; e < 8; ++e) {
    int c = 0;
    if (s > 0.0f && s < INFINITY) c = max(-127, min(127, __float2int_rn(__fdiv_rn(bf16lo(w[0]), s))));
    out |= static_cast<unsigned long long>(c & 0xFF) << (8 * e);
    w[0] = __funnelshift_r(w[0], w[1], 16); w[1] = __funnelshift_r(w[1], w[2], 16); w[2] = __funnelshift_r(w[2], w[3], 16); w[3] >>= 16;
  }
  return make_uint2(static_cast<uint32_t>(out), static_cast<uint32_t>(out >> 32));
}

// What no new row points at: lengths of sequences without new tokens, and offsets that fall or go past the rows that there are.  By CTAs of
// their own behind those of the rows, so that it lengthens nobody's chain of loads.
constexpr int kCheckedBy = 1024;            // sequences a CTA looks at
__device__ __forceinline__ void check_sequences(const AppendParams& p, int cta) {
  const int first = cta * kCheckedBy, last = min(p.B, first + kCheckedBy);
  bool bad = false;
  for (int b = first + static_cast<int>(threadIdx.x); b < last; b += kAppendThreads) {
    const int32_t len = p.seqlens[b];
    const int64_t begin = p.cu[b], end = p.cu[b + 1];
    bad = bad || len < 0 || len > p.cap || begin < 0 || end < begin || end - begin > len || end > p.n_rows;
  }
  if (bad) atomicMax(p.status, kStatusBadShape);
}

constexpr int kAppendCtas = 7;              // resident on an SM at least
template <bool kInt8, int kVecs>            // kVecs: 16-byte pieces of a BF16 row a lane holds (rows of up to 128 kVecs values)
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas)
kv_append_kernel(const __grid_constant__ AppendParams p) {
  const int lane = threadIdx.x & 31, half = lane >> 4, hl = lane & 15;
  const int64_t warps = static_cast<int64_t>(p.row_ctas) * (kAppendThreads / 32);
  pdl_wait_primary();
  pdl_launch_dependents();
  if (static_cast<int>(blockIdx.x) >= p.row_ctas) {
    check_sequences(p, blockIdx.x - p.row_ctas);
    return;
  }
  const int D = half ? p.c.Dv : p.c.D;
  const uint16_t* src = half ? p.v_new : p.k_new;
  const int64_t src_ld = half ? p.v_ld : p.k_ld;
  const PagedRows rows = half ? p.c.v : p.c.k, scales = half ? p.c.vs : p.c.ks;
  const int64_t items = p.n_rows * p.head_groups;
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * (kAppendThreads / 32) + (threadIdx.x >> 5); item < items; item += warps) {
    const int64_t n = item / p.head_groups;
    const int g0 = static_cast<int>(item - n * p.head_groups) * p.heads, g1 = min(p.c.Hkv, g0 + p.heads);
    constexpr int kAhead = kVecs == 1 ? 4 : 2;         // heads whose rows are under way together
    uint4 x[kAhead][kVecs];
    auto fetch = [&](int h, uint4 (&v)[kVecs]) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int d = (i * 16 + hl) * 8;
        v[i] = make_uint4(0, 0, 0, 0);
        if (h < g1 && d < D) v[i] = __ldcs(reinterpret_cast<const uint4*>(src + n * src_ld + static_cast<int64_t>(h) * D + d));
      }
    };
#pragma unroll
    for (int a = 0; a < kAhead; ++a) fetch(g0 + a, x[a]);
    const int b = sequence_of(p.cu, p.B, n, lane);
    if (b < 0) continue;
    const int32_t len = p.seqlens[b];
    const int32_t begin = p.cu[b], end = p.cu[b + 1];
    const int64_t pos = static_cast<int64_t>(len) - end + n;
    // (a sequence with more new tokens than tokens gets none of them; the last term is for a cu that falls)
    if (len > p.cap || static_cast<int64_t>(end) - begin > len || pos < 0 || pos >= len) {
      if (lane == 0) atomicMax(p.status, kStatusBadShape);
      continue;
    }
    const uint32_t page = div_by(static_cast<uint32_t>(pos), p.c.page), slot = static_cast<uint32_t>(pos) - page * p.c.page.d;
    const int32_t blk = p.table[static_cast<int64_t>(b) * p.max_blocks + page];
    if (static_cast<uint32_t>(blk) >= static_cast<uint64_t>(p.c.num_blocks)) {
      if (lane == 0) atomicMax(p.status, kStatusBadShape);
      continue;
    }
    uint8_t* dst = rows.base + row_offset(rows, blk, slot);
    uint8_t* dst_s = kInt8 ? scales.base + row_offset(scales, blk, slot) : nullptr;
    for (int h = g0; h < g1; h += kAhead) {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (h + a >= g1) break;
        uint8_t* to = dst + (h + a) * rows.head;
        if constexpr (!kInt8) {
#pragma unroll
          for (int i = 0; i < kVecs; ++i) {
            const int d = (i * 16 + hl) * 8;
            if (d < D) *reinterpret_cast<uint4*>(to + d * 2) = x[a][i];
          }
        } else {
          uint32_t top = 0;                              // (as bits, where a NaN is above infinity: a maximum of floats would drop it)
#pragma unroll
          for (int i = 0; i < kVecs; ++i) top = max(top, __float_as_uint(unit_absmax(x[a][i])));
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
          const float m = __uint_as_float(top);
          float s = by_127(m), inv;
          const bool plain = m > 1e-28f && m < 1e32f;
          if (!plain) s = __fdiv_rn(m, 127.0f);
          asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(m));
          inv *= 127.0f;
#pragma unroll
          for (int i = 0; i < kVecs; ++i) {
            const int d = (i * 16 + hl) * 8;
            if (d < D) *reinterpret_cast<uint2*>(to + d) = plain ? codes_of(x[a][i], s, inv) : codes_by_division(x[a][i], s);
          }
          if (hl == 0) *reinterpret_cast<float*>(dst_s + (h + a) * scales.head) = s;
        }
        if (p.weights && lane == 0) p.weights[(static_cast<int64_t>(b) * p.c.Hkv + h + a) * p.ld + pos] = 0.0f;
      }
      if (h + kAhead < g1) {
#pragma unroll
        for (int a = 0; a < kAhead; ++a) fetch(h + kAhead + a, x[a]);
      }
    }
  }
}

template <bool kInt8, int kVecs>
msd_status_t launch_append(AppendParams& p, cudaStream_t s) {
  const int64_t per = kAppendThreads / 32, ctas = (p.n_rows * p.head_groups + per - 1) / per, most = 64LL * sm_count();
  p.row_ctas = static_cast<int>(ctas < most ? ctas : most);
  const int check_ctas = (p.B + kCheckedBy - 1) / kCheckedBy;
  return launch_pdl(kv_append_kernel<kInt8, kVecs>, dim3(p.row_ctas + check_ctas), dim3(kAppendThreads), 0, s, option(OPT_NO_PDL) != 1, p) == cudaSuccess
             ? MSD_OK
             : (cudaGetLastError(), MSD_ERR_CUDA);
}

// ---------------------------------------------------------------------------------------------------------------------------
// Eviction, first kernel: which tokens stay.  A cluster of CTAs per (sequence, KV head) holds the weights as ordered integers in
// registers (16 a thread at most; longer rows are read again in each pass) and finds the k-th largest in up to three passes: the range that
// holds it, at first from the smallest key to the largest, is cut into 2048 bins, a histogram of it is made in shared memory, added up over
// the cluster by remote atomics on what is not zero (integers: the order does not matter), and a scan from the top gives the bin that
// is the next range.  (Cutting the range that is there, not the whole range of the bits, spreads the first histogram over more bins: threads
// that add to the same one wait for each other.)  What is above the k-th stays, of what
// equals it the first ones; a scan over the positions in order gives each its new place.  (Finding it by two bits a round, three counts
// over all keys: 61 instead of 17 us for 256 rows of 2048 to 8192, which are 16 since keys are walked four at a time.  The peers' histograms read, not added to by atomics: 8 rows of 131072
// 48 -> 52 us, the move included.)
// ---------------------------------------------------------------------------------------------------------------------------
struct EvictParams {
  PagedCache c;
  const int32_t *table, *dst_table, *seqlens;
  const float* weights;
  int64_t ld, new_ld, cap, dst_cap;
  int max_blocks, dst_max_blocks, B, budget, recent, sinks;
  int32_t *new_seqlens, *kept;
  float* new_weights;
  int warp_rows, chunks;             // of the move: rows of a warp, CTAs of a (sequence, KV head)
  unsigned* status;
};

__device__ __forceinline__ int evict_len(const EvictParams& p, int b) {
  const int32_t n = p.seqlens[b];
  return static_cast<int>(min(static_cast<int64_t>(n < 0 ? 0 : n), p.cap));
}

// Order of the weights as unsigned integers: NaN above the others, -0 as 0.  0 is no key, and kProtected that of a token that stays anyway.
constexpr uint32_t kProtected = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return kProtected - 1;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t caddr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(caddr) : "memory");
  return v;
}
__device__ __forceinline__ void add_cluster_u32(uint32_t caddr, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(caddr), "r"(v) : "memory");
}

__device__ __forceinline__ void count_shared(uint32_t saddr) {
  asm volatile("red.relaxed.cta.shared::cta.add.u32 [%0], 1;" ::"r"(saddr) : "memory");
}

constexpr int kBins = 2048, kPasses = 3;
constexpr uint32_t kNowhere = 0xFFFFFFFFu;

template <int kKeys, int kSelThreads>        // keys a thread keeps; 0: none, they are read from memory in every pass
__global__ void __launch_bounds__(kSelThreads, kSelThreads == 128 ? 6 : 1024 / kSelThreads)
kv_evict_select_kernel(const __grid_constant__ EvictParams p, int cluster_ctas) {
  const int ctas = kSelThreads > 128 ? cluster_ctas : 1;
  constexpr int kSelWarps = kSelThreads / 32, kBinsEach = kBins / kSelThreads;
  __shared__ __align__(16) uint32_t own[kBins];          // histogram of this CTA's keys
  __shared__ __align__(16) uint32_t all[kSelThreads > 128 ? kPasses : 1][kSelThreads > 128 ? kBins : 1];      // of the cluster's, a pass each (128 threads: no cluster)
  __shared__ uint32_t range[2];                         // smallest and largest key of this CTA
  __shared__ uint32_t part[kSelWarps][2];
  __shared__ uint32_t found[3];                         // bin, keys above it, keys in it
  __shared__ uint32_t totals[2];                        // staying for sure, equal to the threshold
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % ctas, bk = blockIdx.x / ctas;
  const int b = bk / p.c.Hkv, hk = bk - b * p.c.Hkv;
  pdl_wait_primary();
  pdl_launch_dependents();
  const int L = evict_len(p, b);
  if (hk == 0 && rank == 0 && threadIdx.x == 0) {
    if (L != p.seqlens[b]) atomicMax(p.status, kStatusBadShape);
    p.new_seqlens[b] = min(L, p.budget);
  }
  const float* w = p.weights + (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.ld;
  float* new_w = p.new_weights + (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.new_ld;
  int32_t* kept = p.kept + (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.budget;
  if (L <= p.budget) {                                  // (alike in all CTAs of the cluster)
    for (int i = rank * kSelThreads + threadIdx.x; i < L; i += ctas * kSelThreads) {
      kept[i] = i;
      new_w[i] = w[i];
    }
    return;
  }
  // Positions in order: CTA by CTA, warp by warp, 32 at a time; lane `lane` of this warp has begin + 32 j.
  const int rows = static_cast<int>((static_cast<uint32_t>(L) + ctas * kSelThreads - 1) / (ctas * kSelThreads));
  const uint32_t begin = (static_cast<uint32_t>(rank) * kSelWarps + warp) * rows * 32 + lane;      // (all of them below 2^32)
  const uint32_t lo = p.sinks, middle = L - p.recent - p.sinks;       // what is not protected: the first one, how many (more than 0)
  const uint32_t want = p.budget;
  // (j-th position of this lane; `there`: how many there are behind `begin`)
  const float* w_lane = w + begin;
  const int there = L - static_cast<int>(min(begin, static_cast<uint32_t>(L)));
  const uint32_t from_lo = begin - lo;
  auto key_of = [&](int j, float x) -> uint32_t { return from_lo + j * 32 < middle ? weight_key(x) : (j * 32 < there ? kProtected : 0u); };
  auto key_at = [&](int j) -> uint32_t { return key_of(j, j * 32 < there ? w_lane[j * 32] : 0.0f); };
  uint32_t key[kKeys > 0 ? kKeys : 1];
  if constexpr (kKeys > 0) {      // (loads side by side: no branch between them)
    float x[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; ++j) x[j] = j < rows && j * 32 < there ? w_lane[j * 32] : 0.0f;
#pragma unroll
    for (int j = 0; j < kKeys; ++j) key[j] = j < rows ? key_of(j, x[j]) : 0u;
  }
  auto for_keys = [&](auto&& f) {                       // (alike in all lanes)
    if constexpr (kKeys > 0) {
#pragma unroll
      for (int j0 = 0; j0 < kKeys; j0 += 4) {           // (key[j] is 0, which counts nowhere, from `rows` on)
        if (j0 >= rows) break;
#pragma unroll
        for (int j = j0; j < j0 + 4; ++j) f(j, key[j]);
      }
    } else {
#pragma unroll 4
      for (int j = 0; j < rows; ++j) f(j, key_at(j));
    }
  };
  uint32_t T = kProtected - 1, above = p.sinks + p.recent;       // the want-th largest key, and how many are above it
  if (want > above) {
    uint32_t smallest = 0xFFFFFFFFu, largest = 0;
    for_keys([&](int, uint32_t k) {
      if (k != 0) smallest = min(smallest, k);
      if (k != kProtected) largest = max(largest, k);
    });
    smallest = __reduce_min_sync(0xffffffffu, smallest);
    largest = __reduce_max_sync(0xffffffffu, largest);
    if (lane == 0) { part[warp][0] = smallest; part[warp][1] = largest; }
    if (kSelThreads > 128 && ctas > 1) {
      for (int i = threadIdx.x; i < kPasses * kBins; i += kSelThreads) (&all[0][0])[i] = 0;
    }
    __syncthreads();
    smallest = __reduce_min_sync(0xffffffffu, part[lane & (kSelWarps - 1)][0]);
    largest = __reduce_max_sync(0xffffffffu, part[lane & (kSelWarps - 1)][1]);
    if (ctas > 1) {
      if (threadIdx.x == 0) { range[0] = smallest; range[1] = largest; }
      __syncwarp();
      cluster_arrive_all();
      cluster_wait_all();
      smallest = __reduce_min_sync(0xffffffffu, ld_cluster_u32(mapa_shared(smem_u32(&range[0]), lane & (ctas - 1))));
      largest = __reduce_max_sync(0xffffffffu, ld_cluster_u32(mapa_shared(smem_u32(&range[1]), lane & (ctas - 1))));
    }
    T = smallest;                                       // the key lies in [T, T + 2^bits)
    int bits = 32 - __clz(largest - smallest);
    const uint32_t own_u = smem_u32(own);
    for (int pass = 0; bits > 0; ++pass) {              // 11 bits fewer each time: three passes at most
      const int shift = max(bits - 11, 0);
      const uint32_t bins = bits < 11 ? 1u << bits : kBins;
      uint32_t c[kBinsEach];                            // this thread's bins
#pragma unroll
      for (int i = 0; i < kBinsEach; ++i) own[threadIdx.x * kBinsEach + i] = 0;
      __syncthreads();
      for_keys([&](int, uint32_t k) {
        const uint32_t bin = (k - T) >> shift;
        if (k >= T && bin < bins && k != kProtected) count_shared(own_u + bin * 4);      // (0 is below T)
      });
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kBinsEach; ++i) c[i] = own[threadIdx.x * kBinsEach + i];
      if (kSelThreads > 128 && ctas > 1) {
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) {
          if (c[i] == 0) continue;
          const uint32_t at = smem_u32(&all[pass][threadIdx.x * kBinsEach + i]);
          for (int r = 0; r < ctas; ++r) add_cluster_u32(mapa_shared(at, r), c[i]);
        }
        cluster_arrive_all();
        cluster_wait_all();
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) c[i] = all[pass][threadIdx.x * kBinsEach + i];
      }
      // keys in the bins of the threads after this one
      uint32_t sum = 0;
#pragma unroll
      for (int i = 0; i < kBinsEach; ++i) sum += c[i];
      uint32_t upto = sum;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_down_sync(0xffffffffu, upto, d);
        if (lane + d < 32) upto += y;
      }
      if (lane == 0) part[warp][0] = upto;
      __syncthreads();
      uint32_t later = lane > warp && lane < kSelWarps ? part[lane][0] : 0u;
      later = __reduce_add_sync(0xffffffffu, later) + upto - sum;
      const uint32_t left = want - above;               // the key is the left-th from the top of these
      if (later < left && left <= later + sum) {
        uint32_t n = later;
#pragma unroll
        for (int i = kBinsEach - 1; i >= 0; --i) {
          if (n < left && n + c[i] >= left) {
            found[0] = threadIdx.x * kBinsEach + i;
            found[1] = n;
            found[2] = c[i];
          }
          n += c[i];
        }
      }
      __syncthreads();
      T += found[0] << shift;
      above += found[1];
      bits = shift;
      if (above + found[2] == want) {                   // the whole bin stays, as a rule after two passes: no need to look into it
        above = want;
        --T;
        break;
      }
    }
  }
  const uint32_t need = want - above;                   // of those equal to T, the first ones

  // Two flags a position: it stays for sure (above T), or it equals T.  Their numbers before a position give its new place.
  auto flags = [&](uint32_t k, unsigned* sure, unsigned* equal) {
    *sure = __ballot_sync(0xffffffffu, k > T);
    *equal = __ballot_sync(0xffffffffu, k == T);
  };
  uint32_t a = 0, e = 0;
  for_keys([&](int, uint32_t k) {
    unsigned ms, me;
    flags(k, &ms, &me);
    a += __popc(ms);
    e += __popc(me);
  });
  __syncthreads();
  if (lane == 0) { part[warp][0] = a; part[warp][1] = e; }
  __syncthreads();
  {
    const uint32_t pa = lane < kSelWarps ? part[lane][0] : 0u, pe = lane < kSelWarps ? part[lane][1] : 0u;
    a = __reduce_add_sync(0xffffffffu, lane < warp ? pa : 0u);
    e = __reduce_add_sync(0xffffffffu, lane < warp ? pe : 0u);
    if (ctas > 1) {
      const uint32_t ta = __reduce_add_sync(0xffffffffu, pa), te = __reduce_add_sync(0xffffffffu, pe);
      if (threadIdx.x == 0) { totals[0] = ta; totals[1] = te; }
      __syncwarp();
      cluster_arrive_all();
      cluster_wait_all();
      a += __reduce_add_sync(0xffffffffu, lane < rank ? ld_cluster_u32(mapa_shared(smem_u32(&totals[0]), lane)) : 0u);
      e += __reduce_add_sync(0xffffffffu, lane < rank ? ld_cluster_u32(mapa_shared(smem_u32(&totals[1]), lane)) : 0u);
      cluster_arrive_all();                             // (nobody leaves while a peer may still read its totals)
    }
  }
  auto place = [&](uint32_t k) -> uint32_t {            // new place of this lane's position, or none
    unsigned ms, me;
    flags(k, &ms, &me);
    const uint32_t pa = a + __popc(ms & lanes_below(lane)), pe = e + __popc(me & lanes_below(lane));
    a += __popc(ms);
    e += __popc(me);
    const uint32_t at = pa + min(pe, need);
    // (below the budget as long as the weights are not changed meanwhile; if they are, nothing outside is written all the same)
    return (((ms >> lane) & 1u) || (((me >> lane) & 1u) && pe < need)) && at < want ? at : kNowhere;
  };
  if constexpr (kKeys > 0) {
    float x[kKeys];
#pragma unroll
    for (int j0 = 0; j0 < kKeys; j0 += 4) {
      if (j0 >= rows) break;
#pragma unroll
      for (int j = j0; j < j0 + 4; ++j) {
        key[j] = place(key[j]);
        x[j] = key[j] != kNowhere ? w_lane[j * 32] : 0.0f;
      }
    }
#pragma unroll
    for (int j0 = 0; j0 < kKeys; j0 += 4) {
      if (j0 >= rows) break;
#pragma unroll
      for (int j = j0; j < j0 + 4; ++j) {
        if (key[j] == kNowhere) continue;
        kept[key[j]] = static_cast<int32_t>(begin + j * 32);
        new_w[key[j]] = x[j];
      }
    }
  } else {
    for (int j = 0; j < rows; ++j) {
      const uint32_t at = place(key_at(j));
      if (at == kNowhere) continue;
      kept[at] = static_cast<int32_t>(begin + j * 32);
      new_w[at] = w_lane[j * 32];
    }
  }
  if (ctas > 1) cluster_wait_all();
}

template <int kKeys, int kThreads>
cudaError_t launch_select(const EvictParams& p, int64_t units, int ctas, cudaStream_t s, bool pdl) {
  return launch_pdl_cluster(kv_evict_select_kernel<kKeys, kThreads>, dim3(static_cast<unsigned>(units * ctas)), dim3(kThreads), 0, s, pdl,
                            static_cast<unsigned>(ctas), p, ctas);
}

// ---------------------------------------------------------------------------------------------------------------------------
// Eviction, second kernel: the kept rows go to their new pages.  Bound: HBM (32 x 8 rows of 2048 INT8 tokens, 281 MB: 49 us, 5.8 TB/s).
// A warp takes up to 32 rows: each lane looks up where one of them is and where it goes, and moves its scales; then kLanes lanes (a power of
// two) copy a row's key and value, 16 bytes at a time, several rows under way.  Sources and destinations never overlap, so the
// order of the copies does not matter.
// ---------------------------------------------------------------------------------------------------------------------------
constexpr int kMoveThreads = 128;

template <bool kInt8, int kLanes>
__global__ void __launch_bounds__(kMoveThreads, 8)
kv_evict_move_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kRowsPer = 32 / kLanes, kAhead = 4;      // rows of a step, steps whose loads are under way together
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int hk = blockIdx.x % p.c.Hkv, bc = blockIdx.x / p.c.Hkv, b = bc / p.chunks;
  const int64_t row0 = static_cast<int64_t>(bc - b * p.chunks) * (kMoveThreads / 32 * p.warp_rows) + warp * p.warp_rows;
  pdl_wait_primary();
  pdl_launch_dependents();
  int n = min(evict_len(p, b), p.budget);
  if (n > p.dst_cap) {
    if (row0 == 0 && lane == 0) atomicMax(p.status, kStatusBadShape);
    n = static_cast<int>(p.dst_cap);
  }
  if (row0 >= n) return;
  const int rows = static_cast<int>(min(static_cast<int64_t>(p.warp_rows), n - row0));
  uint32_t ko = 0, vo = 0, kd = 0, vd = 0;               // offsets of this lane's row in units of 16 bytes: from, to
  bool ok = false;
  if (lane < rows) {
    const int i = static_cast<int>(row0) + lane;
    const int32_t from = p.kept[(static_cast<int64_t>(b) * p.c.Hkv + hk) * p.budget + i];
    const bool known = static_cast<uint32_t>(from) < static_cast<uint64_t>(p.cap);       // (not if the weights were changed meanwhile)
    const uint32_t from_page = div_by(known ? from : 0, p.c.page), to_page = div_by(i, p.c.page);
    const int32_t blk = known ? p.table[static_cast<int64_t>(b) * p.max_blocks + from_page] : -1, to = p.dst_table[static_cast<int64_t>(b) * p.dst_max_blocks + to_page];
    const uint32_t slot = from - from_page * p.c.page.d, to_slot = i - to_page * p.c.page.d;
    if (static_cast<uint32_t>(blk) < static_cast<uint64_t>(p.c.num_blocks) && static_cast<uint32_t>(to) < static_cast<uint64_t>(p.c.num_blocks)) {
      ok = true;
      ko = static_cast<uint32_t>(row_offset(p.c.k, blk, slot) >> 4);
      vo = static_cast<uint32_t>(row_offset(p.c.v, blk, slot) >> 4);
      kd = static_cast<uint32_t>(row_offset(p.c.k, to, to_slot) >> 4);
      vd = static_cast<uint32_t>(row_offset(p.c.v, to, to_slot) >> 4);
      if constexpr (kInt8) {
        const float ks = *reinterpret_cast<const float*>(p.c.ks.base + hk * p.c.ks.head + row_offset(p.c.ks, blk, slot));
        const float vs = *reinterpret_cast<const float*>(p.c.vs.base + hk * p.c.vs.head + row_offset(p.c.vs, blk, slot));
        *reinterpret_cast<float*>(p.c.ks.base + hk * p.c.ks.head + row_offset(p.c.ks, to, to_slot)) = ks;
        *reinterpret_cast<float*>(p.c.vs.base + hk * p.c.vs.head + row_offset(p.c.vs, to, to_slot)) = vs;
      }
    } else {
      atomicMax(p.status, kStatusBadShape);
    }
  }
  const int sub = lane / kLanes, l16 = lane % kLanes * 16, es = kInt8 ? 1 : 2;
  const uint32_t oks = __ballot_sync(0xffffffffu, ok) >> sub;
  const uint32_t k_rows = l16 < p.c.D * es ? oks : 0u, v_rows = l16 < p.c.Dv * es ? oks : 0u;      // (bit r: row r + sub)
  uint8_t* kat = p.c.k.base + hk * p.c.k.head + l16;
  uint8_t* vat = p.c.v.base + hk * p.c.v.head + l16;
  for (int r0 = 0; r0 < rows; r0 += kRowsPer * kAhead) {
    uint4 k[kAhead], v[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int r = r0 + a * kRowsPer;                   // (below 32: r0 is a multiple of kRowsPer kAhead, which divides 32 or is more)
      if (r >= 32) break;
      const uint32_t fk = __shfl_sync(0xffffffffu, ko, r + sub), fv = __shfl_sync(0xffffffffu, vo, r + sub);
      if ((k_rows >> r) & 1u) k[a] = __ldcs(reinterpret_cast<const uint4*>(kat + static_cast<uint64_t>(fk) * 16));
      if ((v_rows >> r) & 1u) v[a] = __ldcs(reinterpret_cast<const uint4*>(vat + static_cast<uint64_t>(fv) * 16));
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int r = r0 + a * kRowsPer;
      if (r >= 32) break;
      const uint32_t tk = __shfl_sync(0xffffffffu, kd, r + sub), tv = __shfl_sync(0xffffffffu, vd, r + sub);
      if ((k_rows >> r) & 1u) *reinterpret_cast<uint4*>(kat + static_cast<uint64_t>(tk) * 16) = k[a];
      if ((v_rows >> r) & 1u) *reinterpret_cast<uint4*>(vat + static_cast<uint64_t>(tv) * 16) = v[a];
    }
  }
}

template <bool kInt8, int kLanes>
cudaError_t launch_move(const EvictParams& p, cudaStream_t s, bool pdl) {
  return launch_pdl(kv_evict_move_kernel<kInt8, kLanes>, dim3(static_cast<unsigned>(p.B) * p.chunks * p.c.Hkv), dim3(kMoveThreads), 0, s, pdl, p);
}

// positions stay below 2^31 - 4096, so that no sum of theirs wraps
inline int64_t position_cap(int64_t blocks, int32_t page) {
  const int64_t n = blocks * page;
  return n < 0x7FFFF000 ? n : 0x7FFFF000;
}

}  // namespace

}  // namespace msd

extern "C" {

msd_status_t msd_kv_append_paged(const void* k_new_bf16, const void* v_new_bf16, int64_t n_rows, int64_t k_ld, int64_t v_ld,
                                 const msd_paged_cache_t* cache, const int32_t* block_table, int32_t max_blocks, const int32_t* seqlens,
                                 const int32_t* cu_new, int32_t B, float* weights, int64_t ld, void* stream) {
  using namespace msd;
  AppendParams p;
  if (const msd_status_t st = paged_cache_view(cache, &p.c)) return st;
  if (B < 0 || B > (1 << 20) || max_blocks < 1 || n_rows < 0 || n_rows > 0x7FFFFFFF || (weights && ld < 1)) return MSD_ERR_BAD_SHAPE;
  if (k_ld < static_cast<int64_t>(cache->Hkv) * cache->D || v_ld < static_cast<int64_t>(cache->Hkv) * cache->Dv) return MSD_ERR_BAD_SHAPE;
  if (B == 0 || n_rows == 0) return MSD_OK;
  if (!k_new_bf16 || !v_new_bf16 || !block_table || !seqlens || !cu_new) return MSD_ERR_NULL_POINTER;
  if (!aligned(k_new_bf16, 16) || !aligned(v_new_bf16, 16) || k_ld % 8 != 0 || v_ld % 8 != 0 || !aligned(block_table, 4) || !aligned(seqlens, 4) ||
      !aligned(cu_new, 4) || !aligned(weights, 4))
    return MSD_ERR_BAD_ALIGNMENT;
  p.status = device_status_ptr();
  if (!p.status) return MSD_ERR_CUDA;
  p.k_new = static_cast<const uint16_t*>(k_new_bf16);
  p.v_new = static_cast<const uint16_t*>(v_new_bf16);
  p.n_rows = n_rows;
  p.k_ld = k_ld;
  p.v_ld = v_ld;
  p.table = block_table;
  p.seqlens = seqlens;
  p.cu = cu_new;
  p.max_blocks = max_blocks;
  p.cap = position_cap(max_blocks, cache->page_size);
  if (weights && p.cap > ld) p.cap = ld;
  p.B = B;
  p.weights = weights;
  p.ld = ld;
  // KV heads a warp takes: as many as leave an item for every warp of the machine, one for a few rows
  p.heads = cache->Hkv;
  while (p.heads > 1 && n_rows * ((cache->Hkv + p.heads - 1) / p.heads) < static_cast<int64_t>(kAppendCtas) * kAppendThreads / 32 * sm_count()) p.heads = (p.heads + 1) / 2;
  p.head_groups = (cache->Hkv + p.heads - 1) / p.heads;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool wide = cache->D > 128 || cache->Dv > 128;
  if (cache->type == MSD_CACHE_INT8) return wide ? launch_append<true, 2>(p, s) : launch_append<true, 1>(p, s);
  return wide ? launch_append<false, 2>(p, s) : launch_append<false, 1>(p, s);
}

msd_status_t msd_kv_evict_paged(const msd_paged_cache_t* cache, const int32_t* block_table, int32_t max_blocks, const int32_t* seqlens,
                                const float* weights, int64_t ld, int32_t B, int32_t budget, int32_t recent, int32_t sinks,
                                const int32_t* dst_block_table, int32_t dst_max_blocks, int32_t* new_seqlens, float* new_weights,
                                int64_t new_ld, int32_t* kept, void* stream) {
  using namespace msd;
  EvictParams p;
  if (const msd_status_t st = paged_cache_view(cache, &p.c)) return st;
  if (B < 0 || B > (1 << 20) || max_blocks < 1 || dst_max_blocks < 1 || ld < 1 || budget < 1 || budget > 0x7FFFF000 || recent < 0 || sinks < 0 ||
      static_cast<int64_t>(recent) + sinks > budget || new_ld < budget)
    return MSD_ERR_BAD_SHAPE;
  if (B == 0) return MSD_OK;
  if (!block_table || !seqlens || !weights || !dst_block_table || !new_seqlens || !new_weights || !kept) return MSD_ERR_NULL_POINTER;
  if (!rows_within(p.c.k, cache->num_blocks, cache->page_size, int64_t{1} << 36) || !rows_within(p.c.v, cache->num_blocks, cache->page_size, int64_t{1} << 36))
    return MSD_ERR_UNSUPPORTED;
  if (block_table == dst_block_table) return MSD_ERR_UNSUPPORTED;
  if (!aligned(block_table, 4) || !aligned(seqlens, 4) || !aligned(weights, 4) || !aligned(dst_block_table, 4) || !aligned(new_seqlens, 4) ||
      !aligned(new_weights, 4) || !aligned(kept, 4))
    return MSD_ERR_BAD_ALIGNMENT;
  // what is written lies in nothing that is read, and nothing is written twice
  const __int128 heads = static_cast<__int128>(B) * cache->Hkv;
  const struct { const void* at; __int128 bytes; } written[] = {{new_seqlens, B * 4LL}, {new_weights, heads * new_ld * 4}, {kept, heads * budget * 4}},
      read[] = {{block_table, B * 4LL * max_blocks}, {dst_block_table, B * 4LL * dst_max_blocks}, {seqlens, B * 4LL}, {weights, heads * ld * 4}};
  for (int i = 0; i < 3; ++i) {
    for (const auto& r : read)
      if (overlap(written[i].at, written[i].bytes, r.at, r.bytes)) return MSD_ERR_UNSUPPORTED;
    for (int j = 0; j < i; ++j)
      if (overlap(written[i].at, written[i].bytes, written[j].at, written[j].bytes)) return MSD_ERR_UNSUPPORTED;
  }
  p.status = device_status_ptr();
  if (!p.status) return MSD_ERR_CUDA;
  p.table = block_table;
  p.dst_table = dst_block_table;
  p.seqlens = seqlens;
  p.weights = weights;
  p.ld = ld;
  p.new_ld = new_ld;
  p.max_blocks = max_blocks;
  p.dst_max_blocks = dst_max_blocks;
  p.cap = position_cap(max_blocks, cache->page_size);
  if (p.cap > ld) p.cap = ld;
  p.dst_cap = position_cap(dst_max_blocks, cache->page_size);
  p.B = B;
  p.budget = budget;
  p.recent = recent;
  p.sinks = sinks;
  p.new_seqlens = new_seqlens;
  p.kept = kept;
  p.new_weights = new_weights;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool pdl = option(OPT_NO_PDL) != 1;

  // CTAs of a cluster: 2048 positions each while the machine is not full, and as many as the longest row needs (8 x 1024 x 16 positions
  // fit; longer rows are read again in every pass).  (16 CTAs, which this device allows, took 4 us more on 8 rows of 131072.)  1024
  // threads where 512 would hold more than 16 keys each: the warps' latencies, not their number, set the pace.
  const int64_t units = static_cast<int64_t>(B) * cache->Hkv;
  if (units > (1 << 24)) return MSD_ERR_UNSUPPORTED;
  int ctas = 1;
  while (ctas < 8 && (p.cap > ctas * 16384LL || (p.cap > ctas * 2048LL && units * ctas <= sm_count()))) ctas *= 2;
  const int64_t keys = (p.cap + ctas * 512LL - 1) / (ctas * 512LL);
  const cudaError_t err = p.cap <= 512   ? launch_select<4, 128>(p, units, 1, s, pdl)
                          : keys <= 4  ? launch_select<4, 512>(p, units, ctas, s, pdl)
                          : keys <= 8  ? launch_select<8, 512>(p, units, ctas, s, pdl)
                          : keys <= 16 ? launch_select<16, 512>(p, units, ctas, s, pdl)
                          : keys <= 32 ? launch_select<16, 1024>(p, units, ctas, s, pdl)
                                       : launch_select<0, 1024>(p, units, ctas, s, pdl);
  if (err != cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }

  // rows of a warp: 32 where that leaves 32 warps to an SM, 8 at least
  const int64_t most = p.cap < budget ? p.cap : budget;
  p.warp_rows = 32;
  while (p.warp_rows > 8 && units * most < 32LL * p.warp_rows * sm_count()) p.warp_rows /= 2;
  const int64_t cta_rows = kMoveThreads / 32 * p.warp_rows, chunks = (most + cta_rows - 1) / cta_rows;
  if (units * chunks > 0x7FFFFFFF) return MSD_ERR_UNSUPPORTED;
  p.chunks = static_cast<int>(chunks);
  const int widest = (cache->D > cache->Dv ? cache->D : cache->Dv) * (cache->type == MSD_CACHE_INT8 ? 1 : 2);      // bytes of a row
  cudaError_t moved;
  if (cache->type == MSD_CACHE_INT8) moved = widest <= 128 ? launch_move<true, 8>(p, s, pdl) : launch_move<true, 16>(p, s, pdl);
  else moved = widest <= 128 ? launch_move<false, 8>(p, s, pdl) : (widest <= 256 ? launch_move<false, 16>(p, s, pdl) : launch_move<false, 32>(p, s, pdl));
  if (moved != cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }
  return MSD_OK;
}

}  // extern "C"
