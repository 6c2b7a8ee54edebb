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
// shuffles away.  The rows are asked for before the warp looks for the sequence and the page they go to.
// ---------------------------------------------------------------------------------------------------------------------------
constexpr int kAppendThreads = 256;

struct AppendParams {
  PagedCache c;
  const uint16_t *k_new, *v_new;
  int64_t n_rows, k_ld, v_ld;
  const int32_t *table, *seqlens, *cu;
  int64_t cap;
  int max_blocks, B;
  int heads, head_groups;       // KV heads a warp takes, groups of them
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

// 8 BF16 values -> 8 codes rne(x / s), bit for bit those of a true division
__device__ __forceinline__ uint2 codes_of(const uint4& v, float s, float inv) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t o[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = (e & 1) ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
    int q;
    if (s > 1e-30f) q = quant_i8(x, s, inv);
    else q = s > 0.0f ? __float2int_rn(__fdiv_rn(x, s)) : 0;
    q = max(-127, min(127, q));
    o[e >> 2] |= static_cast<uint32_t>(q & 0xFF) << (8 * (e & 3));
  }
  return make_uint2(o[0], o[1]);
}

template <bool kInt8, int kVecs>            // kVecs: 16-byte pieces of a BF16 row a lane holds (rows of up to 128 kVecs values)
__global__ void __launch_bounds__(kAppendThreads)
kv_append_kernel(const __grid_constant__ AppendParams p) {
  const int lane = threadIdx.x & 31, half = lane >> 4, hl = lane & 15;
  const int64_t warps = static_cast<int64_t>(gridDim.x) * (kAppendThreads / 32);
  pdl_wait_primary();
  pdl_launch_dependents();
  const int D = half ? p.c.Dv : p.c.D;
  const uint16_t* src = half ? p.v_new : p.k_new;
  const int64_t src_ld = half ? p.v_ld : p.k_ld;
  const PagedRows rows = half ? p.c.v : p.c.k, scales = half ? p.c.vs : p.c.ks;
  const int64_t items = p.n_rows * p.head_groups;
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * (kAppendThreads / 32) + (threadIdx.x >> 5); item < items; item += warps) {
    const int64_t n = item / p.head_groups;
    const int g0 = static_cast<int>(item - n * p.head_groups) * p.heads, g1 = min(p.c.Hkv, g0 + p.heads);
    constexpr int kAhead = 4;               // heads whose rows are under way together
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
          float m = 0.0f;
#pragma unroll
          for (int i = 0; i < kVecs; ++i) m = fmaxf(m, unit_absmax(x[a][i]));
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          const float s = __fdiv_rn(m, 127.0f), inv = __frcp_rn(s);
#pragma unroll
          for (int i = 0; i < kVecs; ++i) {
            const int d = (i * 16 + hl) * 8;
            if (d < D) *reinterpret_cast<uint2*>(to + d) = codes_of(x[a][i], s, inv);
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
msd_status_t launch_append(const AppendParams& p, cudaStream_t s) {
  const int64_t per = kAppendThreads / 32, ctas = (p.n_rows * p.head_groups + per - 1) / per, most = 8LL * sm_count();
  return launch_pdl(kv_append_kernel<kInt8, kVecs>, dim3(static_cast<unsigned>(ctas < most ? ctas : most)), dim3(kAppendThreads), 0, s,
                    option(OPT_NO_PDL) != 1, p) == cudaSuccess
             ? MSD_OK
             : (cudaGetLastError(), MSD_ERR_CUDA);
}

// ---------------------------------------------------------------------------------------------------------------------------
// Eviction, first kernel: which tokens stay.  A cluster of CTAs per (sequence, KV head) holds the weights as ordered integers in
// registers (32 a thread at most; longer rows are read again each round) and finds the k-th largest by two bits a round: three counts,
// summed over the warps and, through the peers' shared memory, over the cluster.  What is above it stays, of what equals it the
// first ones; a scan over the positions in order gives each its new place.
// ---------------------------------------------------------------------------------------------------------------------------
constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;

struct EvictParams {
  PagedCache c;
  const int32_t *table, *dst_table, *seqlens;
  const float* weights;
  int64_t ld, new_ld, cap, dst_cap;
  int max_blocks, dst_max_blocks, B, budget, recent, sinks;
  int32_t *new_seqlens, *kept;
  float* new_weights;
  int rows_per_cta, chunks;          // of the move
  unsigned* status;
};

__device__ __forceinline__ int evict_len(const EvictParams& p, int b) {
  const int32_t n = p.seqlens[b];
  return static_cast<int>(min(static_cast<int64_t>(n < 0 ? 0 : n), p.cap));
}

// order of the weights as unsigned integers: NaN above everything, -0 as 0; never 0
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t caddr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(caddr) : "memory");
  return v;
}

template <int kKeys>        // keys a thread keeps; 0: none, they are read from memory in every round
__global__ void __launch_bounds__(kSelThreads)
kv_evict_select_kernel(const __grid_constant__ EvictParams p, int ctas) {
  __shared__ uint32_t part[kSelWarps][3];
  __shared__ uint32_t sums[2][3];                       // this CTA's counts, by round parity
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
  const int rows = (L + ctas * kSelThreads - 1) / (ctas * kSelThreads);
  const int64_t begin = (static_cast<int64_t>(rank) * kSelWarps + warp) * rows * 32 + lane;
  const int lo = p.sinks, hi = L - p.recent;            // what is not protected
  const uint32_t want = static_cast<uint32_t>(p.budget - p.sinks - p.recent);
  auto key_at = [&](int j) -> uint32_t {
    const int64_t i = begin + j * 32;
    return i >= lo && i < hi ? weight_key(w[i]) : 0u;
  };
  uint32_t key[kKeys > 0 ? kKeys : 1];
  if constexpr (kKeys > 0) {
#pragma unroll
    for (int j = 0; j < kKeys; ++j) key[j] = j < rows ? key_at(j) : 0u;
  }
  auto for_keys = [&](auto&& f) {                       // (alike in all lanes)
    if constexpr (kKeys > 0) {
#pragma unroll
      for (int j = 0; j < kKeys; ++j)
        if (j < rows) f(j, key[j]);
    } else {
#pragma unroll 4
      for (int j = 0; j < rows; ++j) f(j, key_at(j));
    }
  };
  // counts of the cluster; every thread of it calls this, with alternating parity
  auto cluster_sum = [&](uint32_t (&c)[3], int parity) {
#pragma unroll
    for (int i = 0; i < 3; ++i) c[i] = __reduce_add_sync(0xffffffffu, c[i]);
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < 3; ++i) part[warp][i] = c[i];
    }
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const uint32_t v = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? part[lane][i] : 0u);
        if (lane == 0) sums[parity][i] = v;
      }
    }
    if (ctas > 1) {
      __syncwarp();
      cluster_arrive_all();
      cluster_wait_all();
#pragma unroll
      for (int i = 0; i < 3; ++i)
        c[i] = __reduce_add_sync(0xffffffffu, lane < ctas ? ld_cluster_u32(mapa_shared(smem_u32(&sums[parity][i]), lane)) : 0u);
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 3; ++i) c[i] = sums[parity][i];
    }
  };

  uint32_t T = 0, above = 0;                            // the want-th largest key, and how many are above it
  if (want > 0) {
    int parity = 0;
    for (int s = 30; s >= 0; s -= 2) {
      const uint32_t t1 = T + (1u << s), t2 = T + (2u << s), t3 = T + (3u << s);
      uint32_t c[3] = {0, 0, 0};
      for_keys([&](int, uint32_t k) {
        c[0] += k >= t1;
        c[1] += k >= t2;
        c[2] += k >= t3;
      });
      cluster_sum(c, parity);
      parity ^= 1;
      if (c[2] >= want) {
        T = t3;
      } else if (c[1] >= want) {
        T = t2;
        above = c[2];
      } else if (c[0] >= want) {
        T = t1;
        above = c[1];
      } else {
        above = c[0];
      }
    }
  }
  const uint32_t need = want - above;                   // of those equal to T, the first ones

  // Two flags a position: it stays for sure (protected, or above T), or it equals T.  Their numbers before a position give its new place.
  auto flags = [&](int j, uint32_t k, unsigned* sure, unsigned* equal) {
    const int64_t i = begin + j * 32;
    *sure = __ballot_sync(0xffffffffu, i < L && (i < lo || i >= hi || (want > 0 && k > T)));
    *equal = __ballot_sync(0xffffffffu, want > 0 && k == T);
  };
  uint32_t a = 0, e = 0;
  for_keys([&](int j, uint32_t k) {
    unsigned ms, me;
    flags(j, k, &ms, &me);
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
  for_keys([&](int j, uint32_t k) {
    unsigned ms, me;
    flags(j, k, &ms, &me);
    const uint32_t pa = a + __popc(ms & lanes_below(lane)), pe = e + __popc(me & lanes_below(lane));
    if (((ms >> lane) & 1u) || (((me >> lane) & 1u) && pe < need)) {
      const int64_t i = begin + j * 32;
      const uint32_t at = pa + min(pe, need);
      kept[at] = static_cast<int32_t>(i);
      new_w[at] = w[i];
    }
    a += __popc(ms);
    e += __popc(me);
  });
  if (ctas > 1) cluster_wait_all();
}

// ---------------------------------------------------------------------------------------------------------------------------
// Eviction, second kernel: the kept rows go to their new pages.  Bound: HBM.  kLanes lanes (a power of two) copy a row's key and value,
// 16 bytes at a time; a warp has 32 / kLanes rows under way, four times over.  Sources and destinations never overlap, so
// the order of the copies does not matter.
// ---------------------------------------------------------------------------------------------------------------------------
constexpr int kMoveThreads = 256;

template <bool kInt8, int kLanes>
__global__ void __launch_bounds__(kMoveThreads)
kv_evict_move_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kRowsPerWarp = 32 / kLanes, kAhead = 4;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int hk = blockIdx.x % p.c.Hkv, bc = blockIdx.x / p.c.Hkv, b = bc / p.chunks;
  const int64_t row0 = static_cast<int64_t>(bc - b * p.chunks) * p.rows_per_cta;
  pdl_wait_primary();
  pdl_launch_dependents();
  int n = min(evict_len(p, b), p.budget);
  if (row0 >= n) return;
  if (n > p.dst_cap) {
    if (threadIdx.x == 0) atomicMax(p.status, kStatusBadShape);
    n = static_cast<int>(p.dst_cap);
  }
  const int end = static_cast<int>(min(static_cast<int64_t>(n), row0 + p.rows_per_cta));
  const int32_t* kept = p.kept + (static_cast<int64_t>(b) * p.c.Hkv + hk) * p.budget;
  const int32_t* table = p.table + static_cast<int64_t>(b) * p.max_blocks;
  const int32_t* dst_table = p.dst_table + static_cast<int64_t>(b) * p.dst_max_blocks;
  const int sub = lane / kLanes, l = lane % kLanes;
  const int es = kInt8 ? 1 : 2;
  const bool has_k = l * 16 < p.c.D * es, has_v = l * 16 < p.c.Dv * es;
  constexpr int kStep = kMoveThreads / 32 * kRowsPerWarp;
  for (int i0 = static_cast<int>(row0) + warp * kRowsPerWarp + sub; i0 - sub < end; i0 += kStep * kAhead) {
    int32_t from[kAhead], blk[kAhead], to[kAhead];
    uint32_t slot[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int i = i0 + a * kStep;
      from[a] = i < end ? kept[i] : -1;
      to[a] = i < end ? dst_table[div_by(i, p.c.page)] : 0;
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      blk[a] = 0;
      slot[a] = 0;
      if (from[a] < 0) continue;
      const uint32_t page = div_by(from[a], p.c.page);
      slot[a] = from[a] - page * p.c.page.d;
      blk[a] = table[page];
    }
    uint4 k[kAhead], v[kAhead];
    float ks[kAhead], vs[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      if (from[a] >= 0 && (static_cast<uint32_t>(blk[a]) >= static_cast<uint64_t>(p.c.num_blocks) ||
                           static_cast<uint32_t>(to[a]) >= static_cast<uint64_t>(p.c.num_blocks))) {
        atomicMax(p.status, kStatusBadShape);
        from[a] = -1;
      }
      if (from[a] < 0) continue;
      if (has_k) k[a] = __ldcs(reinterpret_cast<const uint4*>(p.c.k.base + hk * p.c.k.head + row_offset(p.c.k, blk[a], slot[a]) + l * 16));
      if (has_v) v[a] = __ldcs(reinterpret_cast<const uint4*>(p.c.v.base + hk * p.c.v.head + row_offset(p.c.v, blk[a], slot[a]) + l * 16));
      if (kInt8 && l == 0) ks[a] = *reinterpret_cast<const float*>(p.c.ks.base + hk * p.c.ks.head + row_offset(p.c.ks, blk[a], slot[a]));
      if (kInt8 && l == 1) vs[a] = *reinterpret_cast<const float*>(p.c.vs.base + hk * p.c.vs.head + row_offset(p.c.vs, blk[a], slot[a]));
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      if (from[a] < 0) continue;
      const int i = i0 + a * kStep;
      const uint32_t s = i - div_by(i, p.c.page) * p.c.page.d;
      if (has_k) *reinterpret_cast<uint4*>(p.c.k.base + hk * p.c.k.head + row_offset(p.c.k, to[a], s) + l * 16) = k[a];
      if (has_v) *reinterpret_cast<uint4*>(p.c.v.base + hk * p.c.v.head + row_offset(p.c.v, to[a], s) + l * 16) = v[a];
      if (kInt8 && l == 0) *reinterpret_cast<float*>(p.c.ks.base + hk * p.c.ks.head + row_offset(p.c.ks, to[a], s)) = ks[a];
      if (kInt8 && l == 1) *reinterpret_cast<float*>(p.c.vs.base + hk * p.c.vs.head + row_offset(p.c.vs, to[a], s)) = vs[a];
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
  // KV heads a warp takes: as many as leave a warp for every place on the machine (64 an SM), one for a few rows
  p.heads = cache->Hkv;
  while (p.heads > 1 && n_rows * ((cache->Hkv + p.heads - 1) / p.heads) < 64LL * sm_count()) p.heads = (p.heads + 1) / 2;
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
  if (block_table == dst_block_table || weights == new_weights || seqlens == new_seqlens) return MSD_ERR_UNSUPPORTED;
  if (!aligned(block_table, 4) || !aligned(seqlens, 4) || !aligned(weights, 4) || !aligned(dst_block_table, 4) || !aligned(new_seqlens, 4) ||
      !aligned(new_weights, 4) || !aligned(kept, 4))
    return MSD_ERR_BAD_ALIGNMENT;
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

  // CTAs of a cluster: 2048 positions each while the machine is not full, and as many as the longest row needs (8 x 512 x 32 positions
  // fit; longer rows are read again in every round)
  const int64_t units = static_cast<int64_t>(B) * cache->Hkv;
  if (units > (1 << 24)) return MSD_ERR_UNSUPPORTED;
  int ctas = 1;
  while (ctas < 8 && (p.cap > static_cast<int64_t>(ctas) * kSelThreads * 32 || (p.cap > ctas * 2048LL && units * ctas * 2 <= 2LL * sm_count()))) ctas *= 2;
  const int64_t keys = (p.cap + static_cast<int64_t>(ctas) * kSelThreads - 1) / (static_cast<int64_t>(ctas) * kSelThreads);
  const dim3 grid(static_cast<unsigned>(units * ctas)), block(kSelThreads);
  const unsigned cluster = static_cast<unsigned>(ctas);
  cudaError_t err;
  if (keys <= 4) err = launch_pdl_cluster(kv_evict_select_kernel<4>, grid, block, 0, s, pdl, cluster, p, ctas);
  else if (keys <= 16) err = launch_pdl_cluster(kv_evict_select_kernel<16>, grid, block, 0, s, pdl, cluster, p, ctas);
  else if (keys <= 32) err = launch_pdl_cluster(kv_evict_select_kernel<32>, grid, block, 0, s, pdl, cluster, p, ctas);
  else err = launch_pdl_cluster(kv_evict_select_kernel<0>, grid, block, 0, s, pdl, cluster, p, ctas);
  if (err != cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }

  // rows of a CTA: 256 where that leaves the machine its CTAs, 32 at least
  const int64_t most = p.cap < budget ? p.cap : budget;
  p.rows_per_cta = 256;
  while (p.rows_per_cta > 32 && units * ((most + p.rows_per_cta - 1) / p.rows_per_cta) < 4LL * sm_count()) p.rows_per_cta /= 2;
  while (units * ((most + p.rows_per_cta - 1) / p.rows_per_cta) > 0x7FFFFFFF) p.rows_per_cta *= 2;
  p.chunks = static_cast<int>((most + p.rows_per_cta - 1) / p.rows_per_cta);
  const int widest = (cache->D > cache->Dv ? cache->D : cache->Dv) * (cache->type == MSD_CACHE_INT8 ? 1 : 2);      // bytes of a row
  if (cache->type == MSD_CACHE_INT8) err = widest <= 128 ? launch_move<true, 8>(p, s, pdl) : launch_move<true, 16>(p, s, pdl);
  else err = widest <= 128 ? launch_move<false, 8>(p, s, pdl) : (widest <= 256 ? launch_move<false, 16>(p, s, pdl) : launch_move<false, 32>(p, s, pdl));
  if (err != cudaSuccess) {
    cudaGetLastError();
    return MSD_ERR_CUDA;
  }
  return MSD_OK;
}

}  // extern "C"
