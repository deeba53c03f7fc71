// Attention of new tokens over a paged cache (phyai_paged_attention): entry point, the kernel for few rows, the fp32 kernel and the
// merge of key ranges.
//
// Row (token i, head h) of a request sees keys [0, limit(i)); o = sum_k p_k v_k / sum_k p_k, p_k = 2^(scale log2(e) (q k_k - max)).
// Statistics and accumulators are fp32; P is rounded to bf16 (off by at most 2^-8 of each weight, as V itself is) because
// it is an operand of the tensor cores; the fp32 cache keeps everything fp32.
//
// Few rows (one token of a request is `group` rows): the cache is read once and nothing is reused, so memory bounds it.  Every warp
// walks 16-key tiles of its own through its own ring of TMA copies, without any barrier between warps:
//   S^T = K Q^T      mma.sync m16n8k16: keys are the 16 rows, 8 query rows the columns, so that 8 rows (pi0: the 8 heads of a token)
//                    fill the instruction; as Q K^T half of it would be empty
//   P^T              transposed in registers (movmatrix) into the B operand of
//   O^T += V^T P^T   V^T by transposing ldmatrix
// The warps of a block merge through shared memory, the blocks of a cluster through distributed shared memory, several clusters of a
// row (key ranges) through a second kernel.
// Measured, one token a request, keys and values from memory (other requests' calls between two of the same): 8 heads of 256, 64 requests of 601 - 969 keys
// 16.5 us, 3.2 TB/s (12.7 where the 51 MB lie in the L2), 256 43 us, 4.8 TB/s, one request of 969 keys 9.3 us (8.4; start, lengths -> pages ->
// copies, cluster merge: a chain of trips to the L2); 8 heads of 128 over 8 x 24576 - 32768 keys 50 us with the merge, 4.7 TB/s.  Figures of variants below: of one
// state over and over, in the L2 as far as it fits.  What lengths cannot do: every row tile gets the same clusters, as the host does not know them; one
// request of 32768 keys among 63 of 800 takes 113 us, four blocks' time, where 64 of 800 take 16.6.
#include <atomic>
#include <cstdio>
#include <cstring>
#include <numeric>

#include "paged.cuh"
#include "attention.cuh"
#include "tc_pair.cuh"
#include "tmap.h"

namespace phyai {
namespace {

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int row, int block, int plane, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(block), "r"(plane), "r"(bar)
      : "memory");
}

// =============================================================================================
// few rows, bf16
// =============================================================================================
constexpr int FW = 4;                    // warps of a block
template <int DH>
struct Few {
  static constexpr int TILE = 16 * DH * 2;                 // 16 keys or values: blocks of 64 channels [DH / 64][16][128 B], swizzled
  static constexpr int SLOTS = 24576 / TILE;               // of a warp's ring: K and V tiles in turn; 96 KB a block, two blocks an SM
  static constexpr int RING = SLOTS * TILE;
  static constexpr size_t SMEM = 1024 + (size_t)FW * RING;
};
constexpr int FEW_LEAST = 2;             // tiles of 16 keys per warp in a range, at least

__device__ __forceinline__ float ld_remote(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_remote4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A cluster of `csize` blocks takes the keys of one range of a row tile, each block a part of them.
template <int DH, int NT>
__global__ void __launch_bounds__(FW * 32, 2) k_paged_few(const PagedAttn a, const __grid_constant__ CUtensorMap map, const int csize) {
  using F = Few<DH>;
  constexpr int RT = 8 * NT, KS = DH / 16, NS = F::SLOTS, PITCH = DH + 4;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[FW][NS];
  __shared__ float s_m[FW][RT], s_l[FW][RT], s_M[RT], s_L[RT];
  __shared__ int abort_flag, s_again[RT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int hk = blockIdx.y, unit = blockIdx.x / csize, rank = blockIdx.x - unit * csize;
  const uint32_t ring0 = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = ring0 + (uint32_t)warp * F::RING;
  pdl_launch_dependents();
  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < NS; ++i) mbar_init(smem_u32(&full[warp][i]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x < RT) s_again[threadIdx.x] = 0;
  __syncthreads();
  pdl_wait();
  const WaitCtx wc{a.status, &abort_flag, a.wait_limit};
  PagedRequest r;
  int tile;
  if (!paged_unit<RT>(a, unit, r, tile)) {
    if (threadIdx.x == 0) paged_raise(a.status, a.pb);
    return;
  }
  if (r.b < 0) return;
  const int rows = min(RT, r.n * a.group - tile * RT), row0 = tile * RT;
  const int n_keys = r.limit((row0 + rows - 1) / a.group, a.causal);              // (limits grow with the row)
  const int tiles = (n_keys + 15) >> 4, ranges = ranges_of(tiles, a.ranges, FEW_LEAST * FW * csize), range = blockIdx.z;
  if (range >= ranges) return;                                                    // (the whole cluster)
  const int c0 = (int)((long long)tiles * range / ranges), c1 = (int)((long long)tiles * (range + 1) / ranges);       // tiles of the cluster, of this block
  const int t0 = c0 + (int)((long long)(c1 - c0) * rank / csize), t1 = c0 + (int)((long long)(c1 - c0) * (rank + 1) / csize);
  const int mine = (t1 - t0 - warp + FW - 1) / FW;                                // tiles t0 + warp, + FW, ...

  // ---- copies: K and V of a tile in turn.  Table entries come 32 tiles at a time, one per lane.
  const size_t trow = (size_t)r.b * a.pb.max_pages;
  int page_of = 0;
  auto fetch_pages = [&](int i0) {
    const int i = i0 + lane;
    page_of = i < mine ? a.pb.table[trow + ((t0 + warp + i * FW) << 4 >> a.pb.page_shift)] : 0;
    if ((unsigned)page_of >= (unsigned)a.pb.n_pages) {
      paged_bad_entry(a.status, a.pb);
      page_of = a.pb.n_pages;                                                     // (past the planes: the copy fills in zeros)
    }
  };
  auto issue = [&](int j) {                                                       // copy j: K (even) or V (odd) of tile j / 2
    const int i = j >> 1;
    if ((i & 31) == 0 && !(j & 1)) fetch_pages(i);
    const int page = __shfl_sync(0xffffffffu, page_of, i & 31);
    if (lane == 0) {
      const int key = (t0 + warp + i * FW) << 4, sl = j % NS;
      const int row = (int)(((long long)page << a.pb.page_shift) + (key & ((1 << a.pb.page_shift) - 1)));
      const uint32_t bar = smem_u32(&full[warp][sl]);
      mbar_expect_tx(bar, F::TILE);
      tma_rows(ring + (uint32_t)sl * F::TILE, &map, row, hk * (DH / 64), a.plane + (j & 1), bar);
    }
  };
  for (int j = 0; j < min(NS, 2 * mine); ++j) issue(j);

  // ---- Q^T as B operand: lane (g, t) holds channels 16 kk + 2 t, + 1 and + 8, + 9 of row g
  uint32_t qf[NT][KS][2];
  int lim[NT][2], min_lim = 0x7fffffff;            // of rows 2 t and 2 t + 1
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rr = nt * 8 + g;
    const bool live = rr < rows;
    const int i = (row0 + rr) / a.group, h = hk * a.group + (row0 + rr) % a.group;
    const uint32_t* qp = reinterpret_cast<const uint32_t*>((const __nv_bfloat16*)a.q + (live ? (r.lo + i) * a.q_stride + (long long)h * DH : 0)) + t;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      qf[nt][kk][0] = live ? qp[kk * 8] : 0u;
      qf[nt][kk][1] = live ? qp[kk * 8 + 4] : 0u;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int re = nt * 8 + 2 * t + e;
      lim[nt][e] = re < rows ? r.limit((row0 + re) / a.group, a.causal) : n_keys;
      min_lim = min(min_lim, lim[nt][e]);
    }
  }
  min_lim = __reduce_min_sync(0xffffffffu, min_lim);

  float acc[NT][KS][4] = {}, m[NT][2], l[NT][2] = {};
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = -INFINITY;
  const int rowk = lane & 15, chk = lane >> 4;                       // ldmatrix of K: keys 0-15, chunks 2 kk, 2 kk + 1
  const int rowv = (lane & 7) + ((lane >> 4) << 3), chv = (lane >> 3) & 1;   // of V: (keys 0-7, ch 0-7), (0-7, 8-15), (8-15, 0-7), (8-15, 8-15)
  for (int it = 0; it < mine; ++it) {
    const int jk = 2 * it, jv = jk + 1, key0 = (t0 + warp + it * FW) << 4;
    const uint32_t ks = ring + (uint32_t)(jk % NS) * F::TILE, vs = ring + (uint32_t)(jv % NS) * F::TILE;
    mbar_wait_drain(smem_u32(&full[warp][jk % NS]), (uint32_t)(jk / NS) & 1u, wc);
    __syncwarp();                                                    // (lanes leave the wait one by one; what follows is of the whole warp)
    float s[NT][2][4] = {};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      uint32_t kf[4];
      const int ch = 2 * kk + chk;
      ldsm_x4(ks + (uint32_t)((ch >> 3) * 2048 + rowk * 128 + (((ch & 7) ^ (rowk & 7)) << 4)), kf[0], kf[1], kf[2], kf[3]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16(s[nt][kk & 1], kf, qf[nt][kk][0], qf[nt][kk][1]);
    }
    __syncwarp();
    if (jk + NS < 2 * mine) issue(jk + NS);
    uint32_t pf[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (s[nt][0][e] + s[nt][1][e]) * a.scale_log2;
      if (key0 + 16 > min_lim) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = key0 + g + (e >> 1) * 8 < lim[nt][e & 1] ? x[e] : -INFINITY;
      }
      float mx[2], corr[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[e] = fmaxf(x[e], x[e + 2]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], o));
        const float mn = fmaxf(m[nt][e], mx[e]), sub = mn == -INFINITY ? 0.f : mn;
        corr[e] = ex2_fast(m[nt][e] - sub);
        x[e] = ex2_fast(x[e] - sub), x[e + 2] = ex2_fast(x[e + 2] - sub);
        l[nt][e] = l[nt][e] * corr[e] + x[e] + x[e + 2];
        m[nt][e] = mn;
      }
      if (__any_sync(0xffffffffu, corr[0] != 1.0f || corr[1] != 1.0f)) {
#pragma unroll
        for (int ct = 0; ct < KS; ++ct) acc[nt][ct][0] *= corr[0], acc[nt][ct][1] *= corr[1], acc[nt][ct][2] *= corr[0], acc[nt][ct][3] *= corr[1];
      }
      pf[nt][0] = transpose8x8(pack_bf16(x[0], x[1]));
      pf[nt][1] = transpose8x8(pack_bf16(x[2], x[3]));
    }
    mbar_wait_drain(smem_u32(&full[warp][jv % NS]), (uint32_t)(jv / NS) & 1u, wc);
    __syncwarp();
    if (key0 + 16 > r.kv) {                                          // rows past the cached tokens hold anything: their values become zeros
      const int keep = r.kv - key0;
      for (int i = lane; i < (16 - keep) * (DH / 8); i += 32) {
        const int row = keep + i / (DH / 8), ch = i % (DH / 8);
        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(vs + (uint32_t)((ch >> 3) * 2048 + row * 128 + (ch & 7) * 16)), "r"(0u) : "memory");
      }
      __syncwarp();
    }
#pragma unroll
    for (int ct = 0; ct < KS; ++ct) {
      uint32_t vf[4];
      const int ch = 2 * ct + chv;
      ldsm_x4_t(vs + (uint32_t)((ch >> 3) * 2048 + rowv * 128 + (((ch & 7) ^ (rowv & 7)) << 4)), vf[0], vf[1], vf[2], vf[3]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16(acc[nt][ct], vf, pf[nt][0], pf[nt][1]);
    }
    __syncwarp();
    if (jv + NS < 2 * mine) issue(jv + NS);
  }

  // ---- the warps' results: rows of DH fp32 (4 more: free of bank conflicts) in each warp's own ring
  static_assert(RT * PITCH * 4 <= F::RING, "a warp's partial result exceeds its ring");
  float* const part0 = reinterpret_cast<float*>(smem_raw + (ring0 - smem_u32(smem_raw)));
  float* const part = part0 + (size_t)warp * (F::RING / 4);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], o);
      if (g == 0) s_m[warp][nt * 8 + 2 * t + e] = m[nt][e], s_l[warp][nt * 8 + 2 * t + e] = l[nt][e];
    }
#pragma unroll
    for (int ct = 0; ct < KS; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[(nt * 8 + 2 * t + (e & 1)) * PITCH + ct * 16 + g + (e >> 1) * 8] = acc[nt][ct][e];
  }
  __syncthreads();
  // (block) the warps' partial results merged, in place of the first
  for (int i = threadIdx.x; i < rows * (DH / 4); i += FW * 32) {
    const int rr = i / (DH / 4), c = (i % (DH / 4)) * 4;
    float M = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < FW; ++k) M = fmaxf(M, s_m[k][rr]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < FW; ++k) {
      const float w = s_m[k][rr] == -INFINITY ? 0.f : ex2_fast(s_m[k][rr] - M);
      sum += w * s_l[k][rr];
      const float4 v = *reinterpret_cast<const float4*>(part0 + (size_t)k * (F::RING / 4) + rr * PITCH + c);
      o.x += w * v.x, o.y += w * v.y, o.z += w * v.z, o.w += w * v.w;
    }
    *reinterpret_cast<float4*>(part0 + rr * PITCH + c) = o;
    if (c == 0) s_M[rr] = M, s_L[rr] = sum;
  }
  // (cluster) each block takes a part of the channels
  if (csize > 1) cluster_sync_all();
  else __syncthreads();
  const bool skip = paged_stopped(a.status, a.pb) || *reinterpret_cast<volatile int*>(&abort_flag);   // (no partial result of a call that has failed)
  for (int i = rank * (FW * 32) + threadIdx.x; i < rows * (DH / 4); i += csize * (FW * 32)) {
    const int rr = i / (DH / 4), c = (i % (DH / 4)) * 4;
    float M = s_M[rr], sum = s_L[rr];
    float4 o;
    if (csize == 1) {
      o = *reinterpret_cast<const float4*>(part0 + rr * PITCH + c);
    } else {
      const uint32_t am = smem_u32(&s_M[rr]), al = smem_u32(&s_L[rr]), ao = ring0 + (uint32_t)(rr * PITCH + c) * 4u;
      float ms[8], ls[8];
      float4 os[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < csize) ms[k] = ld_remote(map_rank(am, k)), ls[k] = ld_remote(map_rank(al, k)), os[k] = ld_remote4(map_rank(ao, k));
      M = -INFINITY, sum = 0.f, o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < csize) M = fmaxf(M, ms[k]);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < csize) {
          const float w = ms[k] == -INFINITY ? 0.f : ex2_fast(ms[k] - M);
          sum += w * ls[k];
          o.x += w * os[k].x, o.y += w * os[k].y, o.z += w * os[k].z, o.w += w * os[k].w;
        }
    }
    if (skip) continue;
    // (0 x infinity and 0 x NaN of keys that this row does not see, or of its own: told apart below)
    if (a.causal && !(fabsf(o.x) + fabsf(o.y) + fabsf(o.z) + fabsf(o.w) < INFINITY)) s_again[rr] = 1;
    const int tok = r.lo + (row0 + rr) / a.group, h = hk * a.group + (row0 + rr) % a.group;
    const bool sees = r.limit((row0 + rr) / a.group, a.causal) > 0;
    if (ranges == 1) {
      const float inv = paged_inv(sum, sees);
      *reinterpret_cast<uint2*>((__nv_bfloat16*)a.out + ((size_t)tok * a.hq + h) * DH + c) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    } else {
      *reinterpret_cast<float4*>(a.part_o + (((size_t)range * a.pb.tokens + tok) * a.hq + h) * DH + c) = o;
    }
    if (c == 0 && a.ranges > 1) a.part_ml[((size_t)range * a.pb.tokens + tok) * a.hq + h] = make_float4(M, sum, (float)ranges, sees ? 1.f : 0.f);
  }
  // no block leaves while another reads its shared memory; and the rows below are written over all channels
  if (csize > 1) cluster_sync_all();
  else __syncthreads();
  if (!a.causal) return;
  for (int rr = warp; rr < rows; rr += FW) {
    if (!s_again[rr]) continue;
    const int i = (row0 + rr) / a.group, hidden = max(c0 * 16, r.limit(i, 1));
    if (!paged_hidden_odd<DH / 32, __nv_bfloat16>(a, r.b, hk, DH, 0, hidden, min(c1 * 16, r.kv))) continue;
    const int tok = r.lo + i, h = hk * a.group + (row0 + rr) % a.group, c = lane * (DH / 32);
    float o[DH / 32], M, sum;
    paged_row_alone<DH>(a, r.b, (const __nv_bfloat16*)a.q + tok * a.q_stride + (long long)h * DH, hk, c0 * 16, min(c1 * 16, r.limit(i, 1)), o, M, sum);
    const bool sees = r.limit(i, 1) > 0;
    const float inv = paged_inv(sum, sees);
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) {
      if (ranges == 1) ((__nv_bfloat16*)a.out)[((size_t)tok * a.hq + h) * DH + c + e] = __float2bfloat16_rn(o[e] * inv);
      else a.part_o[(((size_t)range * a.pb.tokens + tok) * a.hq + h) * DH + c + e] = o[e];
    }
    if (lane == 0 && ranges > 1) a.part_ml[((size_t)range * a.pb.tokens + tok) * a.hq + h] = make_float4(M, sum, (float)ranges, sees ? 1.f : 0.f);
  }
}

// =============================================================================================
// fp32
// =============================================================================================
constexpr int XK = 32;                   // keys per tile

// A warp takes RW rows, a block NW warps.  Logits: a lane takes one of a tile's 32 keys, so that a load of K is read by all lanes at full width and the queries'
// are broadcasts (with 8 keys a load, repeated for 4 rows, shared memory bounded the kernel at a third of the rate); P V: a lane takes DH / 32
// channels, P are the broadcasts.  The next tile's K is on its way while P V of this one is computed, its V under the next logits; a tile's
// rows in the planes are looked up once, a tile ahead.
// Measured: four requests of 17 tokens over 33 - 81 keys 8.8 us, 10.6 - 12 from memory (the chain of a tile or two); one token over 8 x 8192 keys, 2 kv heads of 128,
// 44 us, 3.0 TB/s; 64 requests of 600 - 968 keys, 8 heads of 256: 56 us, 1.8 TB/s (every pair of rows reads the tile from shared memory; a row a warp
// 48 and 62, four rows a warp 42 and 57, for 42 and 54 then); four chunks of 512 tokens over 2048 keys 20 TFLOP/s, a quarter of the FMA rate: eight warps an SM,
// in step through four barriers a tile.
template <int DH, int RW, int NW>
__global__ void __launch_bounds__(NW * 32) k_paged_f32(const PagedAttn a) {
  constexpr int XT = NW * 32, RT = NW * RW, PITCH = DH + 4, PP = XK + 4, C = DH / 32, CV = C < 4 ? C : 4, CJ = C / CV, RB = RW < 4 ? RW : 4;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ long long s_at[2][XK];        // element offset of a tile's keys in the planes, -1: none
  __shared__ int s_skip;
  float* const Q = reinterpret_cast<float*>(smem_raw);
  float *const K = Q + RT * PITCH, *const V = K + XK * PITCH, *const P = V + XK * PITCH;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hk = blockIdx.y;
  pdl_launch_dependents();
  pdl_wait();
  // (the word is read by one thread: it may go up at any time, and a block whose threads had read different values would go on with some of
  // them, into barriers and shuffles of all.  On its way beside the lengths; looked at behind the first barrier.)
  const int word = tid == 0 ? *reinterpret_cast<const volatile int*>(a.status) : ST_OK;
  PagedRequest r;
  int tile;
  if (!paged_unit<RT>(a, blockIdx.x, r, tile)) {
    if (tid == 0) paged_raise(a.status, a.pb);
    return;
  }
  if (r.b < 0) return;
  const int rows = min(RT, r.n * a.group - tile * RT), row0 = tile * RT;
  const int n_keys = r.limit((row0 + rows - 1) / a.group, a.causal);
  const int tiles = (n_keys + XK - 1) / XK, ranges = ranges_of(tiles, a.ranges, 1), range = blockIdx.z;
  if (range >= ranges) return;
  const int t0 = (int)((long long)tiles * range / ranges), t1 = (int)((long long)tiles * (range + 1) / ranges);
  bool bad_page = false;
  auto look_up = [&](int kt) {
    if (tid < XK && kt < t1) {
      const int key = kt * XK + tid;
      long long row = -1;
      if (key < n_keys) {
        row = paged_row(a.pb, r.b, key);
        bad_page |= row < 0;
      }
      s_at[kt & 1][tid] = row < 0 ? -1 : (row * a.hkv + hk) * DH;
    }
  };
  auto fetch = [&](int kt, const void* plane, float* dst) {
    if (kt < t1) {
#pragma unroll 8
      for (int i = tid; i < XK * (DH / 4); i += XT) {
        const int kr = i / (DH / 4), c = (i % (DH / 4)) * 4;
        const long long at = s_at[kt & 1][kr];
        cp_async16(smem_u32(dst + kr * PITCH + c), (const float*)plane + (at < 0 ? 0 : at + c), at < 0 ? 0u : 16u);
      }
    }
    cp_async_commit();
  };
  look_up(t0);
  if (tid == 0) s_skip = word != ST_OK && paged_stopped(a.status, a.pb);
  __syncthreads();
  if (s_skip) return;
  fetch(t0, a.k_plane, K);
  fetch(t0, a.v_plane, V);
  for (int i = tid; i < RT * (DH / 4); i += XT) {
    const int rr = i / (DH / 4), c = (i % (DH / 4)) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (rr < rows) v = *reinterpret_cast<const float4*>((const float*)a.q + (r.lo + (row0 + rr) / a.group) * a.q_stride + (long long)(hk * a.group + (row0 + rr) % a.group) * DH + c);
    *reinterpret_cast<float4*>(Q + rr * PITCH + c) = v;
  }
  const int wr = warp * RW;                // first row of this warp
  float acc[RW][C] = {}, m[RW], l[RW] = {};            // l: of this lane's keys
  int lim[RW];
#pragma unroll
  for (int i = 0; i < RW; ++i) m[i] = -INFINITY, lim[i] = wr + i < rows ? r.limit((row0 + wr + i) / a.group, a.causal) : n_keys;
  for (int kt = t0; kt < t1; ++kt) {
    look_up(kt + 1);
    cp_async_wait<1>();
    __syncthreads();                       // K of this tile, Q
    float s[RW] = {};
#pragma unroll 4
    for (int d = 0; d < DH; d += 4) {
      const float4 k = *reinterpret_cast<const float4*>(K + lane * PITCH + d);
#pragma unroll
      for (int i = 0; i < RW; ++i) {
        const float4 q = *reinterpret_cast<const float4*>(Q + (wr + i) * PITCH + d);
        s[i] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s[i]))));
      }
    }
    __syncthreads();
    fetch(kt + 1, a.k_plane, K);
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      s[i] = kt * XK + lane < lim[i] ? s[i] * a.scale_log2 : -INFINITY;
      const float mn = fmaxf(m[i], warp_max(s[i])), sub = mn == -INFINITY ? 0.f : mn, p = exp2f(s[i] - sub);
      P[(wr + i) * PP + lane] = p;
      if (mn != m[i]) {                    // (the same in all lanes)
        const float corr = exp2f(m[i] - sub);
        l[i] *= corr, m[i] = mn;
#pragma unroll
        for (int e = 0; e < C; ++e) acc[i][e] *= corr;
      }
      l[i] += p;
    }
    cp_async_wait<1>();
    __syncthreads();                       // V of this tile
#pragma unroll 1
    for (int k = 0; k < XK; k += 4) {
      float v[4][C];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int j = 0; j < CJ; ++j) {
          const float* src = V + (k + kk) * PITCH + lane * CV + 32 * CV * j;
          if constexpr (CV == 4) *reinterpret_cast<float4*>(&v[kk][4 * j]) = *reinterpret_cast<const float4*>(src);
          else *reinterpret_cast<float2*>(&v[kk][2 * j]) = *reinterpret_cast<const float2*>(src);
        }
#pragma unroll
      for (int i0 = 0; i0 < RW; i0 += RB) {
        float p[RB][4];
#pragma unroll
        for (int i = 0; i < RB; ++i) *reinterpret_cast<float4*>(p[i]) = *reinterpret_cast<const float4*>(P + (wr + i0 + i) * PP + k);
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int e = 0; e < C; ++e) acc[i0 + i][e] = fmaf(p[i][kk], v[kk][e], acc[i0 + i][e]);
      }
    }
    __syncthreads();
    fetch(kt + 1, a.v_plane, V);
  }
  cp_async_wait<0>();
  if (bad_page) paged_bad_entry(a.status, a.pb);
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    if (wr + i >= rows) continue;          // (the whole warp)
    const float sum = warp_sum(l[i]);
    const int it = (row0 + wr + i) / a.group, tok = r.lo + it, h = hk * a.group + (row0 + wr + i) % a.group;
    const size_t slot = ((size_t)range * a.pb.tokens + tok) * a.hq + h;
    float* const dst = ranges == 1 ? (float*)a.out + ((size_t)tok * a.hq + h) * DH : a.part_o + slot * DH;
    const float inv = ranges > 1 ? 1.0f : paged_inv(sum, lim[i] > 0);
    float fin = 0.f;
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      float o[CV];
#pragma unroll
      for (int e = 0; e < CV; ++e) o[e] = acc[i][CV * j + e] * inv, fin = fmaf(acc[i][CV * j + e], 0.f, fin);
      if constexpr (CV == 4) *reinterpret_cast<float4*>(dst + lane * 4 + 128 * j) = make_float4(o[0], o[1], o[2], o[3]);
      else *reinterpret_cast<float2*>(dst + lane * 2 + 64 * j) = make_float2(o[0], o[1]);
    }
    if (lane == 0 && a.ranges > 1) a.part_ml[slot] = make_float4(m[i], sum, (float)ranges, lim[i] > 0 ? 1.f : 0.f);
    // (0 x infinity and 0 x NaN: see k_paged_few)
    if (!a.causal || __all_sync(0xffffffffu, fin == 0.f)) continue;
    const int lm = r.limit(it, 1);
    if (!paged_hidden_odd<DH / 32, float>(a, r.b, hk, DH, 0, max(t0 * XK, lm), min(t1 * XK, n_keys))) continue;
    float o[DH / 32], M, sm;
    paged_row_alone<DH>(a, r.b, (const float*)a.q + tok * a.q_stride + (long long)h * DH, hk, t0 * XK, min(t1 * XK, lm), o, M, sm);
    const float w = ranges > 1 ? 1.0f : paged_inv(sm, lm > 0);
    __syncwarp();                          // (behind the stores above, of other lanes)
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) dst[lane * (DH / 32) + e] = o[e] * w;
    if (lane == 0 && ranges > 1) a.part_ml[slot] = make_float4(M, sm, (float)ranges, lm > 0 ? 1.f : 0.f);
  }
}

// =============================================================================================
// merge of key ranges
// =============================================================================================
// A warp per row: weights 2^(m_r - max m), in the order of the ranges; a lane takes DH / 32 channels, four ranges' loads at a time.
template <int DH, typename OUT>
__global__ void __launch_bounds__(128) k_paged_merge(const PagedAttn a) {
  constexpr int C = DH / 32, V = C < 4 ? C : 4;             // channels of a lane, of a load
  const int lane = threadIdx.x & 31, c = lane * C;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5), rows = (long long)a.pb.tokens * a.hq;
  pdl_launch_dependents();
  pdl_wait();
  if (row >= rows) return;
  const int tok = (int)(row / a.hq);
  // (the lengths and the word say whether there is anything in the workspace; its entries are on their way meanwhile)
  const bool mine = !paged_stopped(a.status, a.pb) && tok >= a.pb.cu[0] && tok < a.pb.cu[a.pb.batch];
  float4 ml = lane < a.ranges ? a.part_ml[(size_t)lane * rows + row] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const float* p = a.part_o + (size_t)row * DH + c;
  float x[4][C];
  auto load = [&](float (&to)[C], int k) {
#pragma unroll
    for (int e = 0; e < C; e += V) {
      if constexpr (V == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + (size_t)k * rows * DH + e);
        to[e] = v.x, to[e + 1] = v.y, to[e + 2] = v.z, to[e + 3] = v.w;
      } else {
        const float2 v = *reinterpret_cast<const float2*>(p + (size_t)k * rows * DH + e);
        to[e] = v.x, to[e + 1] = v.y;
      }
    }
  };
  load(x[0], 0), load(x[1], 1);                             // (where a row has ranges it has two; a.ranges > 1: there is memory to read)
  if (!__all_sync(0xffffffffu, mine)) return;               // (the warp as one: the word may change under it)
  // (bounded: where the word was up for the kernel before and is not now, the workspace holds anything)
  const int ranges = min((int)__shfl_sync(0xffffffffu, ml.z, 0), a.ranges);
  if (ranges <= 1) return;
  const bool sees = __shfl_sync(0xffffffffu, ml.w, 0) != 0.f;
  float4 ml2 = make_float4(-INFINITY, 0.f, 0.f, 0.f);       // (up to 64 ranges)
  if (lane + 32 < ranges) ml2 = a.part_ml[(size_t)(lane + 32) * rows + row];
  if (lane >= ranges) ml = make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const float M = warp_max(fmaxf(ml.x, ml2.x));
  const float w1 = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M), w2 = ml2.x == -INFINITY ? 0.f : exp2f(ml2.x - M);
  const float sum = warp_sum(w1 * ml.y + w2 * ml2.y);
  float o[C] = {};
  for (int k0 = 0; k0 < ranges; k0 += 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (k0 + j < ranges && (k0 > 0 || j >= 2)) load(x[j], k0 + j);
      if (k0 + j >= ranges) {
#pragma unroll
        for (int e = 0; e < C; ++e) x[j][e] = 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float w = __shfl_sync(0xffffffffu, k0 + j < 32 ? w1 : w2, (k0 + j) & 31);      // (0 past the ranges)
#pragma unroll
      for (int e = 0; e < C; ++e) o[e] = fmaf(w, x[j][e], o[e]);
    }
  }
  const float inv = paged_inv(sum, sees);
  OUT* dst = (OUT*)a.out + row * DH + c;
#pragma unroll
  for (int e = 0; e < C; e += 2) {
    if constexpr (sizeof(OUT) == 4) *reinterpret_cast<float2*>(dst + e) = make_float2(o[e] * inv, o[e + 1] * inv);
    else *reinterpret_cast<uint32_t*>(dst + e) = pack_bf16(o[e] * inv, o[e + 1] * inv);
  }
}

// =============================================================================================
// host side
// =============================================================================================
std::atomic<unsigned> g_wait_limit{1u << 22};      // of the kernels' waits on copies and MMAs (phyai_paged_set_option)

phyai_status_t bad_arg(const char* m) {
  snprintf(g_paged_err, sizeof(g_paged_err), "%s", m);
  return PHYAI_ERR_INVALID_ARG;
}

template <typename K>
cudaError_t allow_smem(K kern, size_t bytes) { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); }

// Clusters of 2^l blocks of k_paged_few that run at a time on the current device (all its forms have the same shared memory; 0: cannot be said).
int few_active(int l) {
  static PerDeviceCount n[4];
  const int v = n[l].get([l] {
    if (allow_smem(k_paged_few<256, 2>, Few<256>::SMEM) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(1024), cfg.blockDim = dim3(FW * 32), cfg.dynamicSmemBytes = Few<256>::SMEM;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 1u << l, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = 1;
    int active = 0;
    return cudaOccupancyMaxActiveClusters(&active, k_paged_few<256, 2>, &cfg) == cudaSuccess ? active : 0;
  });
  return v > 0 ? v : 0;
}

// What a call launches: the kernel's row tile, its units and key ranges.
struct Plan {
  int f32, pair, rt, ranges, csize;      // csize: blocks of a cluster, which share a range
  long long units;
};
Plan make_plan(const phyai_paged_cache_t* c, int hq, int tokens, int batch, int max_pages, int n_sm) {
  Plan p{};
  p.csize = 1;
  const int group = hq / (int)c->n_kv_heads, holders = tokens < batch ? tokens : batch;      // requests with tokens, at most
  const long long rows = (long long)tokens * group;
  p.f32 = c->dtype == PHYAI_F32;
  const long long keys = (long long)max_pages * c->page_size;
  // More than 16 packed rows a request: the tensor cores' kernel, whose tiles of 256 rows cost what a tile's keys cost to fetch.  The average is
  // all that the host knows, and a chunk beside single tokens is not the average: 63 single tokens over 1000 keys with a chunk of 65, 8 heads of 256,
  // 36 us here, with one of 66 (the other kernel) 25; the chunk over 16000 keys 117 and 83.  21 single tokens over 700 keys: 16.7 and 18.1.
  if (!p.f32 && rows > 16ll * holders && paged_pair_supported((int)c->head_dim, group)) {
    const int per = paged_pair_tokens(group), pairs = paged_pair_resident((int)c->head_dim);
    const long long full = (tokens + per - 1) / per > holders ? (tokens + per - 1) / per : holders;
    p.pair = 1, p.units = (tokens + (per - 1ll) * holders) / per;
    // Key ranges where there are fewer units than one and a half rounds of the pairs, and where the time that splitting saves could be more than
    // it costs (the kernel cuts the keys by the lengths, or leaves the units whole: this is the same rule at the longest that they can be).
    // As many as a unit of three times the average length can have.
    const long long u = full * c->n_kv_heads, tiles = (keys + 127) / 128, rounds = (u + pairs - 1) / pairs;
    long long ranges = 2 * u < 3ll * pairs && tiles * (rounds * pairs - u) > (long long)PAGED_PAIR_MERGE * pairs ? (3ll * pairs + u - 1) / u : 1;
    if (ranges > keys / 256 + 1) ranges = keys / 256 + 1;
    p.ranges = (int)(ranges < 1 ? 1 : ranges > 64 ? 64 : ranges);
    return p;
  }
  if (p.f32) {
    // tiles of 64 rows where there are enough of them for the SMs (17 tokens of 4 heads of 4 requests: 16-row tiles)
    p.rt = rows / 64 * c->n_kv_heads >= n_sm ? 64 : rows <= 4ll * holders ? 4 : rows <= 8ll * holders ? 8 : 16;
  } else {
    p.rt = rows <= 8ll * holders ? 8 : 16;
  }
  // A request's rows are a multiple of the group, so that its last tile misses rt - gcd(rt, group) rows at most.  (A tile more for each request: a grid
  // with 64 empty units beside the 64 of one token of 8 heads each, 12.8 us for 12.5.)
  p.units = (rows + (p.rt - std::gcd(p.rt, group)) * (long long)holders) / p.rt;
  const long long full = (rows + p.rt - 1) / p.rt > holders ? (rows + p.rt - 1) / p.rt : holders, blocks = full * c->n_kv_heads;
  if (p.f32) {
    // Parts of a row tile's keys: five blocks an SM, of at least a tile of 32 (two: 1.5 times the time with one token a request)
    long long parts = (5ll * n_sm + blocks - 1) / blocks;
    if (parts > keys / 32) parts = keys / 32;
    p.ranges = (int)(parts < 1 ? 1 : parts > 64 ? 64 : parts);
    return p;
  }
  // A row tile's keys go to the largest cluster, of up to eight blocks with at least 128 keys each, that lets all tiles run at a time, and to as many of those
  // (key ranges, merged by a second kernel) as run at a time.  What does is asked of the device: 296 blocks, but 33 clusters of eight (one more and its keys
  // wait for a whole round: 18 requests of 4000 - 5000 keys, two clusters each, 27.1 us for 19.0 with one; 36 of 600 - 969 keys 19.4 for 11.9 with
  // four blocks each; 256 of one block each 41, of two 49).  Clusters before ranges: 64 requests 12.5 us for 14.8 and more.
  int most = few_active(0);
  for (int l = 1; l <= 3 && (128ll << l) <= keys && blocks <= few_active(l); ++l) p.csize = 1 << l, most = few_active(l);
  long long ranges = most / blocks;
  if (ranges > keys / (128 * p.csize)) ranges = keys / (128 * p.csize);
  p.ranges = (int)(ranges < 1 ? 1 : ranges > 64 ? 64 : ranges);
  return p;
}
size_t partial_bytes(const Plan& p, int hq, int dh, int tokens) {
  return p.ranges > 1 ? (size_t)p.ranges * tokens * hq * ((size_t)dh * 4 + 16) + 16 : 0;      // (16: the accumulators begin on 32 bytes)
}

template <int DH, int NT>
cudaError_t launch_few(const PagedAttn& a, const Plan& p, const CUtensorMap& map, cudaStream_t st) {
  static PerDeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = allow_smem(k_paged_few<DH, NT>, Few<DH>::SMEM);
    if (e != cudaSuccess) return e;
    once.done();
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)p.units * p.csize, a.hkv, p.ranges), cfg.blockDim = dim3(FW * 32), cfg.dynamicSmemBytes = Few<DH>::SMEM, cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization, at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = p.csize, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
  cfg.attrs = at, cfg.numAttrs = p.csize > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_paged_few<DH, NT>, a, map, p.csize);
}
template <int DH, int RW, int NW>
cudaError_t launch_f32(const PagedAttn& a, const Plan& p, cudaStream_t st) {
  constexpr size_t smem = ((size_t)(NW * RW + 2 * XK) * (DH + 4) + NW * RW * (XK + 4)) * 4;
  static PerDeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = allow_smem(k_paged_f32<DH, RW, NW>, smem);
    if (e != cudaSuccess) return e;
    once.done();
  }
  return launch_pdl(k_paged_f32<DH, RW, NW>, dim3((unsigned)p.units, a.hkv, p.ranges), dim3(NW * 32), smem, st, a);
}
}  // namespace

bool paged_pool_map(void* map, const phyai_paged_cache_t* c, uint32_t rows, uint32_t blocks) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return false;
  const cuuint64_t row = (cuuint64_t)c->n_kv_heads * c->head_dim * 2, n = c->n_pages * c->page_size;
  const cuuint64_t dims[4] = {64, n, row / 128, 2ull * c->n_layers}, strides[3] = {row, 128, n * row};
  const cuuint32_t bx[4] = {64, rows, blocks, 1}, es[4] = {1, 1, 1, 1};
  return enc(reinterpret_cast<CUtensorMap*>(map), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, c->pages, dims, strides, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace phyai

extern "C" {

phyai_status_t phyai_paged_set_option(const char* key, int64_t value) {
  using namespace phyai;
  if (!key || strcmp(key, "wait_limit")) return bad_arg("unknown option");
  if (value < 1 || value > (1ll << 30)) return bad_arg("wait_limit must be 1..2^30");
  g_wait_limit.store((unsigned)value, std::memory_order_relaxed);
  return PHYAI_OK;
}

size_t phyai_paged_attention_workspace_bytes(const phyai_paged_cache_t* cache, uint32_t n_q_heads, uint32_t tokens, uint32_t batch,
                                             uint32_t max_pages) {
  using namespace phyai;
  const int n_sm = paged_sm_count();
  // (0 for calls that phyai_paged_attention refuses)
  if (!cache || !cache->n_kv_heads || !n_q_heads || n_q_heads % cache->n_kv_heads || !tokens || !batch || batch > (uint32_t)PAGED_MAX_BATCH || n_sm <= 0) return 0;
  if ((uint64_t)tokens * (n_q_heads / cache->n_kv_heads) > 0x7fffffffull || (uint64_t)max_pages * cache->page_size > PAGED_MAX_KEYS) return 0;
  return partial_bytes(make_plan(cache, (int)n_q_heads, (int)tokens, (int)batch, (int)max_pages, n_sm), (int)n_q_heads, (int)cache->head_dim, (int)tokens);
}

phyai_status_t phyai_paged_attention(const phyai_paged_cache_t* cache, uint32_t layer, uint32_t n_q_heads, uint32_t tokens, const void* q,
                                     uint64_t q_stride, uint32_t batch, const int32_t* cu_q_lens, const int32_t* kv_lens,
                                     const int32_t* page_table, uint32_t max_pages, uint32_t causal, const int32_t* prefix_lens, float scale,
                                     void* out, void* workspace, size_t workspace_bytes, int32_t* status_word, void* stream) {
  using namespace phyai;
  PagedAttn a{};
  const phyai_status_t s = check_paged(cache, layer, batch, cu_q_lens, kv_lens, page_table, max_pages, tokens, false, &a.pb);
  if (s != PHYAI_OK) return s;
  if (!status_word || (tokens && (!q || !out))) return bad_arg("a pointer argument is NULL");
  if (!n_q_heads || n_q_heads % cache->n_kv_heads || n_q_heads > 65535u) return bad_arg("n_q_heads must be a multiple of the cache's n_kv_heads");
  if (prefix_lens && !causal) return bad_arg("prefix_lens without the causal mask");
  if (!(scale >= 0.f) || scale > 1e30f) return bad_arg("scale must be positive (0: 1 / sqrt(head_dim))");
  const uint64_t es = cache->dtype == PHYAI_F32 ? 4 : 2;
  if (q_stride < (uint64_t)n_q_heads * cache->head_dim || q_stride > (1ull << 40)) return bad_arg("a row stride is smaller than the row's heads, or too large");
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(workspace)) & 15u) || (q_stride * es) % 16)
    return bad_arg("pointers and row strides must be multiples of 16 bytes");
  if (((reinterpret_cast<uintptr_t>(status_word) | reinterpret_cast<uintptr_t>(prefix_lens)) & 3u)) return bad_arg("status_word and prefix_lens must be 4-byte aligned");
  if ((uint64_t)tokens * (n_q_heads / cache->n_kv_heads) > 0x7fffffffull) return bad_arg("tokens too large");
  if (!tokens) return PHYAI_OK;
  auto overlap = [&](const void* p, uint64_t bytes) {      // out and what is read
    const uint64_t o = reinterpret_cast<uintptr_t>(out), i = reinterpret_cast<uintptr_t>(p);
    return o < i + bytes && i < o + (uint64_t)tokens * n_q_heads * cache->head_dim * es;
  };
  if (overlap(q, ((tokens - 1ull) * q_stride + (uint64_t)n_q_heads * cache->head_dim) * es) ||
      overlap(cache->pages, 2ull * cache->n_layers * cache->n_pages * cache->page_size * cache->n_kv_heads * cache->head_dim * es))
    return bad_arg("out overlaps q or the pages");
  const int n_sm = paged_sm_count();
  if (n_sm <= 0) {
    snprintf(g_paged_err, sizeof(g_paged_err), "no CUDA device (there is no CPU fallback)");
    return PHYAI_ERR_CUDA;
  }
  const int dh = (int)cache->head_dim;
  const Plan p = make_plan(cache, (int)n_q_heads, (int)tokens, (int)batch, (int)max_pages, n_sm);
  const size_t need = partial_bytes(p, (int)n_q_heads, dh, (int)tokens);
  if (need && (!workspace || workspace_bytes < need)) {
    snprintf(g_paged_err, sizeof(g_paged_err), "needs %zu bytes of workspace, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    return PHYAI_ERR_INVALID_ARG;
  }
  const size_t plane = (size_t)cache->n_pages * cache->page_size * cache->n_kv_heads * dh * es;
  a.q = q, a.q_stride = (long long)q_stride, a.out = out, a.plane = (int)layer * 2;
  a.k_plane = (const char*)cache->pages + 2 * (size_t)layer * plane, a.v_plane = (const char*)a.k_plane + plane;
  a.prefix_lens = prefix_lens, a.causal = causal ? 1 : 0, a.hq = (int)n_q_heads, a.hkv = (int)cache->n_kv_heads, a.group = a.hq / a.hkv;
  a.scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)dh)) * LOG2E;
  a.ranges = p.ranges, a.status = status_word, a.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
  a.part_ml = reinterpret_cast<float4*>(workspace), a.part_o = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(a.part_ml + (size_t)p.ranges * tokens * n_q_heads) + 31) & ~(uintptr_t)31);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = paged_call(status_word, &a.pb);
  if (e != cudaSuccess) {
    snprintf(g_paged_err, sizeof(g_paged_err), "status notes: %s", cudaGetErrorString(e));
    return PHYAI_ERR_CUDA;
  }
  if (p.f32) {
#define PHYAI_F32_ROWS(DH) (p.rt == 4 ? launch_f32<DH, 2, 2>(a, p, st) : p.rt == 8 ? launch_f32<DH, 2, 4>(a, p, st) : p.rt == 16 ? launch_f32<DH, 2, 8>(a, p, st) : launch_f32<DH, 8, 8>(a, p, st))
    e = dh == 64 ? PHYAI_F32_ROWS(64) : dh == 128 ? PHYAI_F32_ROWS(128) : PHYAI_F32_ROWS(256);
#undef PHYAI_F32_ROWS
  } else if (p.pair) {
    e = launch_paged_pair(a, cache, p.units * a.hkv * p.ranges, st);
  } else {
    CUtensorMap map;
    if (!paged_pool_map(&map, cache, 16, cache->head_dim / 64)) {
      snprintf(g_paged_err, sizeof(g_paged_err), "cuTensorMapEncodeTiled failed");
      return PHYAI_ERR_CUDA;
    }
    if (dh == 64) e = p.rt == 8 ? launch_few<64, 1>(a, p, map, st) : launch_few<64, 2>(a, p, map, st);
    else if (dh == 128) e = p.rt == 8 ? launch_few<128, 1>(a, p, map, st) : launch_few<128, 2>(a, p, map, st);
    else e = p.rt == 8 ? launch_few<256, 1>(a, p, map, st) : launch_few<256, 2>(a, p, map, st);
  }
  if (e == cudaSuccess && p.ranges > 1) {
    const dim3 grid((unsigned)(((long long)tokens * n_q_heads + 3) / 4));
    if (p.f32) e = dh == 64 ? launch_pdl(k_paged_merge<64, float>, grid, dim3(128), 0, st, a) : dh == 128 ? launch_pdl(k_paged_merge<128, float>, grid, dim3(128), 0, st, a) : launch_pdl(k_paged_merge<256, float>, grid, dim3(128), 0, st, a);
    else e = dh == 64 ? launch_pdl(k_paged_merge<64, __nv_bfloat16>, grid, dim3(128), 0, st, a) : dh == 128 ? launch_pdl(k_paged_merge<128, __nv_bfloat16>, grid, dim3(128), 0, st, a) : launch_pdl(k_paged_merge<256, __nv_bfloat16>, grid, dim3(128), 0, st, a);
  }
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) {
    snprintf(g_paged_err, sizeof(g_paged_err), "paged attention launch failed: %s", cudaGetErrorString(e));
    return PHYAI_ERR_CUDA;
  }
  return PHYAI_OK;
}

}  // extern "C"
