// Attention of many new tokens over a paged cache: a persistent grid of CTA pairs (tcgen05 cta_group::2).
//
// A pair takes a unit: 2 x 128 packed rows (each CTA floor(128 / group) tokens of a request with the query heads of one kv head) and
// walks the keys that any of them sees, then goes on to its next unit without leaving the pipeline: the next unit's operands are on their way
// and its first logits go through the softmax while the accumulator of the last one is read out.
//   S = Q K^T   M = 256, N = 128 keys, K = head_dim; Q and K in shared memory; two S buffers (head_dim 128: three) in tensor memory
//   softmax     four threads per row, straight from tensor memory; P (bf16) over the S buffer; the accumulator
//               is rescaled only when a maximum grows by more than 2^8 (the old one is kept otherwise: exact algebra)
//   O += P V    M = 256, N = head_dim, K = 128 keys; P is the tensor-memory A operand, V an MN-major B operand
// K: CTA h of the pair fetches block h (64 keys) of a tile, V: its half of the channels of both blocks; the tensor cores read the other
// half from the peer, so that every SM fetches and reads half of a tile: with one CTA per 128 rows the shared memory (Q 128 + K 128 rows
// per product, at 128 bytes a clock) would bound the products.  All operands come by tensor-map copies, keys and values piece by piece:
// a piece is the rows of a page, 64 at most, one lane of the loading warp per copy.  Rows past the cached tokens may hold anything: their
// logits are masked by index, their values overwritten with zeros in shared memory (0 x NaN); pieces of pages that a request does not have
// are fetched from past the pool, which fills in zeros.  Keys inside a tile that a row does not see (causal) may hold infinities, too:
// rows whose result is not finite are looked at again after the last unit (see paged_row_alone).
//
// Few units (short chunks over long histories): all tiles in a row, an equal part for each pair; the fp32 results of a unit's key ranges are
// merged by k_paged_merge.  (Units cut into equal ranges of their own, about two for each pair: 71 for 66.5 us below, for some pairs had a fifth more.)
// Warps of a CTA: 0 fetches K and Q, 1 V; 2 goes through the units; 3 issues the MMAs (leader CTA); 4-19 softmax, correction, output.  Every
// wait is bounded; after a give-up the protocol runs to its end and only the global stores are skipped.
//
// Measured, all operands from memory: eight prefixes of 968 tokens (8 heads of 256, one kv head) 69 - 71 us, 0.9 PFLOP/s (SM clock about 1.6 GHz, the power cap); four chunks of
// 384 - 512 tokens over 4096 - 8192 keys (8 heads of 128, two kv heads) 63.8 us with the merge, 0.7 PFLOP/s; eight prefixes with 16 heads of 64 75 us.
// What bounds it, by clocks taken in the kernel: head_dim 256: a tile takes 2150 clocks, of which the products 2048; a unit's end 3700
// to 5600, in which its output goes out and the next one's queries come in through the L2 on all SMs at a time (starting the pairs apart: 71 us
// for 68); four rounds of units where 3.35 would do.  head_dim 128: a tile takes 2050, the products 1024 of it: the chain logits -> maximum (400) ->
// powers (1270; the special-function unit alone 1024) -> P published (60) -> next logits (290), by all four warps of a scheduler at a time; 9700 from
// the end of the kernel before to the first logits, 6000 for the last unit's results.
#include <cstdio>

#include "paged.cuh"
#include "attention.cuh"
#include "attention_choice.h"
#include "tc_pair.cuh"

namespace phyai {
namespace {

constexpr int KB = 128;                        // keys per tile: two blocks of 64
constexpr int PP_THREADS = 20 * 32;
constexpr int PAIR_LEAST = 2;                  // tiles of keys of a pair where units are split, at least

// head_dim 64: V counts as 128 channels, of which the second CTA's half is zero and never fetched (half of 64 channels would be 64 bytes a
// key, another operand layout; the products are not what bounds that head_dim).
template <int DH>
struct PpLayout {
  static constexpr int VN = DH < 128 ? 128 : DH;             // columns of the accumulator
  static constexpr int KBLOCK = 64 * 128;                    // 64 channels of 64 keys
  static constexpr int PIECE = (VN / 128) * KBLOCK;          // V: 64 keys, this CTA's half of the channels
  static constexpr int KTILE = (DH / 64) * KBLOCK;           // K: this CTA's block of 64 keys
  static constexpr int VTILE = 2 * PIECE;                    // V: both blocks
  static constexpr int QTILE = 128 * DH * 2;
  static constexpr int STG = 1024;                           // output staging of a warp: 32 rows x 16 columns
  static constexpr int NB = (512 - VN) / 128;                // buffers of logits: what the accumulator leaves of the 512 columns
  static constexpr size_t USED = 1024 + NB * (size_t)(KTILE + VTILE) + QTILE + 16 * STG;
  // One CTA an SM, and no other kernel that could wait there for tensor memory: two pairs of different kernels, each with tensor memory
  // on one SM and waiting for the other's, would wait for good.
  static constexpr size_t SMEM = USED > 209 * 1024 ? USED : 209 * 1024;
};

__device__ __forceinline__ void copy4d(uint32_t dst, const CUtensorMap* map, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}

// Four MMAs of K = 16 in a row (64 channels, or 64 keys), by the lane with `elected` (one election per product, no branch between
// them: what a warp issues between two MMAs is what bounds it here).  `first`: the first one overwrites the accumulator.
__device__ __forceinline__ void umma2_ss_x4(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t first, uint32_t elected) {
  asm volatile(
      "{\n.reg .pred e, p, q;\n.reg .b64 a1, a2, a3, b1, b2, b3;\n"
      "setp.ne.b32 e, %5, 0;\nsetp.eq.b32 p, %4, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "add.s64 a1, %1, 2;\nadd.s64 b1, %2, 2;\nadd.s64 a2, %1, 4;\nadd.s64 b2, %2, 4;\nadd.s64 a3, %1, 6;\nadd.s64 b3, %2, 6;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], a1, b1, %3, q;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], a2, b2, %3, q;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], a3, b3, %3, q;\n}" ::"r"(d),
      "l"(da), "l"(db), "r"(idesc), "r"(first), "r"(elected)
      : "memory");
}
__device__ __forceinline__ void umma2_ts_x4(uint32_t d, uint32_t ta, uint64_t db, uint32_t idesc, uint32_t first, uint32_t elected) {
  asm volatile(
      "{\n.reg .pred e, p, q;\n.reg .b32 a1, a2, a3;\n.reg .b64 b1, b2, b3;\n"
      "setp.ne.b32 e, %5, 0;\nsetp.eq.b32 p, %4, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "add.s32 a1, %1, 8;\nadd.s64 b1, %2, 128;\nadd.s32 a2, %1, 16;\nadd.s64 b2, %2, 256;\nadd.s32 a3, %1, 24;\nadd.s64 b3, %2, 384;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], [a1], b1, %3, q;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], [a2], b2, %3, q;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], [a3], b3, %3, q;\n}" ::"r"(d),
      "r"(ta), "l"(db), "r"(idesc), "r"(first), "r"(elected)
      : "memory");
}

__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Waits of the pipeline: one instruction in which the warp is suspended until the phase completes, and a call where that takes long.  (The bounded
// polling loop inline at every wait is code, and code is time here: the warp that issues the MMAs shares its scheduler's instruction
// cache with four softmax warps.)
__device__ __noinline__ void wait_long(uint32_t bar, uint32_t parity, const WaitCtx* c) { mbar_wait_drain(bar, parity, *c); }
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, const WaitCtx& c) {
  if (!mbar_try(bar, parity)) wait_long(bar, parity, &c);
}
__device__ __forceinline__ void wait_warp(uint32_t bar, uint32_t parity, const WaitCtx& c) {      // by a whole warp
  wait(bar, parity, c);
  __syncwarp();
}
// index of a buffer in a ring of N and the parity of its phase
template <int N>
struct Ring {
  int at = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void next() {
    if (++at == N) at = 0, parity ^= 1u;
  }
};

// the two loading warps: the first keys and queries go ahead of the first values
__device__ __forceinline__ void first_copies() { asm volatile("bar.sync 1, 64;" ::: "memory"); }
// the four warps that share the rows of a tensor-memory lane quarter
__device__ __forceinline__ void rows_sync(int q) { asm volatile("bar.sync %0, 128;" ::"r"(4 + q) : "memory"); }

// Softmax of a tile of 128 keys, four threads per row (lane quarter q, column part g; 32 columns each, the first `vis` of which the row
// sees; not `live`: a row of no token, whatever it holds): P = 2^(scale S - m) over the logits, as bf16 pairs, 16 columns per part.  m: running maximum (log2 units) of the row, l: sum over
// this thread's columns, acc: the accumulator's rows of this warp, rescaled when the maximum grows; `prev_done` returns once every P V so far
// has completed.  P is published by halves of the keys, and the product of the first 64 starts with the first half alone, over all channels: the
// warps of a quarter, which rescale a fourth of the channels each, meet behind that.
// The special-function unit (16 a clock and SM) takes 1024 clocks of a tile's 2050 to 2150.  (Not faster: a quarter or half of the powers by a
// polynomial on the FMA pipe, 1.04 and 1.10 times the kernel's time; two floats an instruction for scale and sum, 0.99 at head_dim 256 and 1.01 at 128;
// with three buffers the maximum of the next tile before the powers of this one, so that the four warps need not meet between the two, 1.05 at
// head_dim 128; one thread per row, 1.3 and more.)  A NaN or +infinity among the logits makes the maximum and so the whole row NaN.
template <int DH, typename PrevDone>
__device__ __forceinline__ void softmax_tile(float& m, float& l, float (*xch)[128], uint32_t sb, uint32_t acc, int g, int q, int row, int vis, bool live, float scale,
                                             PrevDone prev_done) {
  float s[32];
  tmem_ld32(sb + (uint32_t)(g * 32), s);
  if (__any_sync(0xffffffffu, vis < 32)) {
    asm volatile("" ::: "memory");            // (a branch: as selects, the instructions below would be issued for every tile)
#pragma unroll
    for (int c = 0; c < 32; ++c) s[c] = c < vis ? s[c] : -INFINITY;
  }
  float mx4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
  for (int c = 4; c < 28; c += 8)
#pragma unroll
    for (int e = 0; e < 4; ++e) mx4[e] = max3_nan(mx4[e], s[c + e], s[c + 4 + e]);
#pragma unroll
  for (int e = 0; e < 4; ++e) mx4[e] = max_nan(mx4[e], s[28 + e]);
  xch[g][row] = max_nan(max3_nan(mx4[0], mx4[1], mx4[2]), mx4[3]);
  rows_sync(q);                               // (also: all parts of these S rows have been read -> P may overwrite them)
  float mx = max_nan(max3_nan(xch[0][row], xch[1][row], xch[2][row]), xch[3][row]) * scale;
  mx = mx < INFINITY ? mx : NAN;
  // keep the old maximum unless the new one exceeds it by more than the threshold (exact algebra, no rescaling)
  float m_new = m;
  if (!(mx <= m + PAIR_RESCALE) || m == -INFINITY) m_new = max_nan(m, mx);
  const bool rescale = live && m_new != m && m != -INFINITY;
  const float corr = rescale ? exp2f(m - m_new) : 1.0f;
  const float nsub = m_new == -INFINITY ? 0.f : -m_new;
  float rs[4] = {0.f, 0.f, 0.f, 0.f};
  uint32_t w[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float e0 = ex2_fast(fmaf(s[2 * e], scale, nsub)), e1 = ex2_fast(fmaf(s[2 * e + 1], scale, nsub));
    rs[e & 1] += e0, rs[2 + (e & 1)] += e1;
    w[e] = pack_bf16(e0, e1);
  }
  tmem_st16u(sb + (uint32_t)(g * 16), w);
  if (__any_sync(0xffffffffu, rescale)) {     // rare: rescale this warp's channels of its rows of the accumulator
    prev_done();
    __syncwarp();
    tc_fence_after();
#pragma unroll 1
    for (int c = g * (DH / 4); c < (g + 1) * (DH / 4); c += 16) {
      float o[16];
      tmem_ld16(acc + (uint32_t)c, o);
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] *= corr;
      tmem_st16(acc + (uint32_t)c, o);
    }
    tmem_st_wait();
    tc_fence_before();
    rows_sync(q);
    tc_fence_after();
  }
  tmem_st_wait();
  tc_fence_before();
  __syncwarp();
  l = l * corr + ((rs[0] + rs[1]) + (rs[2] + rs[3]));
  m = m_new;
}

struct alignas(16) Unit {
  PagedRequest r;      // r.b < 0: none
  int hk, tok0;        // first of the unit's tokens in the request
  int t0, T;           // tiles of 128 keys: first, how many (one at least: without a key all of it is masked)
  int range, ranges;
  int pad;
};
constexpr int SPLIT_UNITS = 640;               // units of a kv head, at most, where they are split (the launch asks for it with one and a half a pair at most)
constexpr int UNITS = 8;                       // units that the scheduling warp is ahead, at most

template <int DH>
__global__ void __launch_bounds__(PP_THREADS, 1) __cluster_dims__(2, 1, 1)
    k_paged_pair(const PagedAttn a, const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmkv, const int piece_shift) {
  using L = PpLayout<DH>;
  constexpr int NB = L::NB;
  constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(KB >> 3) << 17) | ((256u >> 4) << 24);
  constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(L::VN >> 3) << 17) | ((256u >> 4) << 24);

  extern __shared__ uint8_t smem_raw[];
  // leader: operands of a buffer complete in both CTAs, P of a buffer (by column half) complete in both, Q complete in both, accumulator
  // read out in both.  Each CTA: logits / P V complete, all logits of a unit complete; own V blocks that are cleared in part.
  __shared__ __align__(8) uint64_t k_full[NB], v_full[NB], p_full[NB][2], q_full, o_free, s_full[NB], pv_done[NB], q_free, v_own, u_full[UNITS], u_free[UNITS];
  __shared__ Unit s_unit[UNITS];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, s_skip;
  __shared__ float xch[2][4][128], xsum[2][4][128];       // what the four threads of a row exchange: maxima (by tile parity), sums (by unit parity)
  __shared__ int s_first[PAGED_MAX_BATCH + 1], s_pos[SPLIT_UNITS + 1], s_list[3];

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int half = blockIdx.x & 1, pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int G = a.group, TOK = 128 / G;                   // tokens of a CTA's 128 rows
  if (tid == 32) prefetch_tmap(&tmkv), prefetch_tmap(&tmq);

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t Ks = base, Vs = base + NB * L::KTILE, Qs = Vs + NB * L::VTILE;
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < NB; ++i) {
      mbar_init(smem_u32(&k_full[i]), 1), mbar_init(smem_u32(&v_full[i]), 2), mbar_init(smem_u32(&p_full[i][0]), 16), mbar_init(smem_u32(&p_full[i][1]), 16);
      mbar_init(smem_u32(&s_full[i]), 1), mbar_init(smem_u32(&pv_done[i]), 1);
    }
    for (int i = 0; i < UNITS; ++i) mbar_init(smem_u32(&u_full[i]), 1), mbar_init(smem_u32(&u_free[i]), half == 0 ? 19 : 18);
    mbar_init(smem_u32(&q_full), 1), mbar_init(smem_u32(&o_free), 32), mbar_init(smem_u32(&q_free), 1), mbar_init(smem_u32(&v_own), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 3) {
    tmem_alloc2(smem_u32(&tmem_slot), 512);
    tc_fence_before();
  }
  if (DH < 128 && half == 1) {
    for (uint32_t i = tid; i < NB * L::VTILE / 16; i += PP_THREADS) asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(Vs + i * 16), "r"(0u) : "memory");
    fence_async_smem();
  }
  __syncthreads();
  pair_sync();                                      // both CTAs' barriers exist before the peer can signal them
  tc_fence_after();
  pdl_launch_dependents();                          // (not before: a later kernel must not take tensor memory that this one still waits for)
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(&tmem_slot), 0);
  const uint32_t tmem_s = tmem_base, tmem_o = tmem_base + NB * KB;
  const WaitCtx wc{a.status, &abort_flag, a.wait_limit, true}, wl = wc;

  // ---- units of each request (both CTAs of a pair read the same lengths and come to the same list)
  pdl_wait();
  if (tid == 0) s_skip = paged_stopped(a.status, a.pb), s_first[0] = 0;
  bool bad = false;
  for (int i = tid; i < a.pb.batch; i += PP_THREADS) {
    const int lo = a.pb.cu[i], hi = a.pb.cu[i + 1], kv = a.pb.kv_lens[i];
    const bool b = paged_entry_bad(a.pb, i, lo, hi, kv, false);
    bad |= b;
    s_first[i + 1] = b ? 0 : (hi - lo + 2 * TOK - 1) / (2 * TOK);
  }
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) paged_raise(a.status, a.pb);
  const bool skip = s_skip != 0;

  // ---- what warp 2 goes by (and, once it has published its last unit, others): s_first: units (of one kv head) before each request; units of one kv
  // head; `each`: 0, or the tiles of a pair where units are split; s_pos: tiles before each unit, of one kv head.
  auto unit_at = [&](int ut) {                      // without a kv head
    Unit u;
    u.hk = u.pad = 0;
    int lo = 0, hi = a.pb.batch;                    // s_first[lo] <= ut < s_first[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_first[mid] <= ut) lo = mid;
      else hi = mid;
    }
    u.r.b = lo, u.r.lo = a.pb.cu[lo], u.r.n = a.pb.cu[lo + 1] - u.r.lo, u.r.kv = a.pb.kv_lens[lo];
    u.r.prefix = a.prefix_lens ? min(max(a.prefix_lens[lo], 0), u.r.kv) : 0;
    u.tok0 = (s_first[lo + 1] - 1 - ut) * 2 * TOK;  // (a request's last, longest unit comes first)
    const int keys = u.r.limit(min(u.tok0 + 2 * TOK, u.r.n) - 1, a.causal);
    u.t0 = 0, u.T = max(1, (keys + KB - 1) / KB), u.range = 0, u.ranges = 1;
    return u;
  };
  // The pair's first unit from `at` on, which moves past it.  Whole units: of every round of n_pairs units one, rounds dealt back and forth;
  // `at` counts rounds.  Split ones: all their tiles in a row, an equal part of it for each pair, so that a pair ends one unit and begins another;
  // `at` is a tile.  A unit of T tiles meets (T - 2) / each + 2 pairs at most: no more than the workspace has room for.
  auto next_unit = [&](int& at, int units, int each) {
    int ut, hk = 0, start = at;
    bool any;
    if (each) {
      const int total = s_pos[units] * a.hkv;
      any = at < (int)min((long long)(pair + 1) * each, (long long)total);
      int lo = 0, hi = units;                       // s_pos[lo] * hkv <= at < s_pos[hi] * hkv
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_pos[mid] * a.hkv <= at) lo = mid;
        else hi = mid;
      }
      ut = lo;
    } else {
      for (;; ++at) {
        ut = at * n_pairs + ((at & 1) ? n_pairs - 1 - pair : pair), any = at * n_pairs < units * a.hkv;
        if (!any || ut < units * a.hkv) break;
      }
      ++at;
      if (a.hkv > 1) hk = ut % a.hkv, ut /= a.hkv;
    }
    if (!any) {
      Unit u{};
      u.r.b = -1, u.T = 0;
      return u;
    }
    Unit u = unit_at(ut);
    u.hk = hk;
    if (each) {
      start = s_pos[ut] * a.hkv;
      if (a.hkv > 1) u.hk = (at - start) / u.T, start += u.hk * u.T;
      const int first = start / each, stop = start + u.T;
      u.range = pair - first, u.ranges = (stop - 1) / each - first + 1;
      u.t0 = at - start;
      at = (int)min((long long)stop, (long long)(pair + 1) * each);
      u.T = at - start - u.t0;
    }
    return u;
  };
  // The units come through shared memory from a warp of their own: some 400 instructions each (searches, divisions), which every warp
  // would else run between its units (20 warps: 2000 clocks of the schedulers' time per unit).
  auto unit = [&](int i) {                          // the i-th unit of this pair, by a whole warp, in turn
    wait_warp(smem_u32(&u_full[i % UNITS]), (uint32_t)(i / UNITS) & 1u, wl);
    const Unit u = s_unit[i % UNITS];
    __syncwarp();
    if (lane == 0) mbar_arrive_local(smem_u32(&u_free[i % UNITS]));
    return u;
  };
  // row of the planes of key `key` of a unit's request; past the pool where the request has no page for it (or a wrong entry)
  const int past = a.pb.n_pages << a.pb.page_shift;
  auto row_of = [&](const PagedRequest& r, int key) {
    if (key >= r.kv) return past;
    const int page = a.pb.table[(size_t)r.b * a.pb.max_pages + (key >> a.pb.page_shift)];
    if ((unsigned)page >= (unsigned)a.pb.n_pages) {
      paged_bad_entry(a.status, a.pb);
      return past;
    }
    return (page << a.pb.page_shift) + (key & ((1 << a.pb.page_shift) - 1));
  };
  const int np = 64 >> piece_shift;                 // pieces of a block of 64 keys
  const int cb = np == 1 ? L::VN / 128 : 1;         // blocks of 64 channels of a copy
  const uint32_t piece_bytes = (uint32_t)(128 << piece_shift);

  if (warp == 0) {
    // =========================== K: a buffer is free again once the logits of the tile NB before exist ==================
    const int nc = np * (DH / 64 / cb), pc = lane % np, ch = (lane / np) * cb;        // copies of a block: one per lane
    int n = 0, i = 0;
    Ring<NB> rg;
    for (Unit u = unit(0); u.r.b >= 0; u = unit(++i)) {
      for (int t = 0; t < u.T; ++t, ++n, rg.next()) {
        const int row = lane < nc ? row_of(u.r, (u.t0 + t) * KB + half * 64 + (pc << piece_shift)) : 0;
        const int bf = rg.at;
        if (n >= NB) wait_warp(smem_u32(&s_full[bf]), rg.parity ^ 1u, wl);
        const uint32_t bar = smem_u32(&k_full[bf]), dst = Ks + (uint32_t)bf * L::KTILE;
        if (half == 0 && lane == 0) mbar_expect_tx(bar, (uint32_t)L::KTILE * 2);
        __syncwarp();
        if (lane < nc) copy4d(dst + (uint32_t)ch * L::KBLOCK + (uint32_t)pc * piece_bytes, &tmkv, row, u.hk * (DH / 64) + ch, a.plane, bar & LEADER_MASK);
        if (t == 0) {                             // Q: its tile is free again once the last logits of the unit before exist
          if (lane == 0) {
            if (i > 0) wait(smem_u32(&q_free), (uint32_t)(i - 1) & 1u, wl);
            if (half == 0) mbar_expect_tx(smem_u32(&q_full), 2 * (uint32_t)(TOK * G * DH * 2));
          }
          __syncwarp();
          if (lane < DH / 64)
            copy4d(Qs + (uint32_t)lane * (128 * 128), &tmq, u.hk * G, u.r.lo + u.tok0 + half * TOK, lane, smem_u32(&q_full) & LEADER_MASK);
          if (n == 0) first_copies();
        }
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // =========================== the pair's units ============================================================================
    int units = 0, each = 0, at = 0;
    if (!bad) {
      for (int i0 = 0; i0 < a.pb.batch; i0 += 32) {
        int n = i0 + lane < a.pb.batch ? s_first[i0 + lane + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, n, o);
          if (lane >= o) n += up;
        }
        if (i0 + lane < a.pb.batch) s_first[i0 + lane + 1] = units + n;
        units += __shfl_sync(0xffffffffu, n, 31);
      }
      __syncwarp();
    }
    if (a.ranges > 1 && units > 0 && units <= SPLIT_UNITS) {
      long long tiles = 0;
      int most = 0;
      for (int i0 = 0; i0 < units; i0 += 32) {
        const int T = i0 + lane < units ? unit_at(i0 + lane).T : 0;
        int n = T;                                  // (32 x 2^24 at most)
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, n, o);
          if (lane >= o) n += up;
        }
        if (i0 + lane < units) s_pos[i0 + lane + 1] = (int)tiles + n;
        tiles += __shfl_sync(0xffffffffu, n, 31), most = max(most, T);
      }
      if (lane == 0) s_pos[0] = 0;
      __syncwarp();
      most = __reduce_max_sync(0xffffffffu, most);
      tiles *= a.hkv;
      // (fp32 results and the second kernel cost what PAGED_PAIR_MERGE tiles do: not where the longest units, left whole, end before that)
      if (tiles <= 0x7fffffff - n_pairs) {
        const int per = ((int)tiles + n_pairs - 1) / n_pairs;
        const long long whole = (long long)most * ((units * a.hkv + n_pairs - 1) / n_pairs);
        if (whole > per + PAGED_PAIR_MERGE) each = max(max(PAIR_LEAST, per), (most - 1) / (a.ranges - 1) + 1);
      }
    }
    if (each) at = (int)min((long long)pair * each, 0x7fffffffll);
    if (lane == 0) s_list[0] = units, s_list[1] = each, s_list[2] = at;
    for (int i = 0;; ++i) {
      const Unit u = next_unit(at, units, each);
      if (i >= UNITS) wait_warp(smem_u32(&u_free[i % UNITS]), (uint32_t)(i / UNITS - 1) & 1u, wl);
      if (lane == 0) {
        s_unit[i % UNITS] = u;
        mbar_arrive_local(smem_u32(&u_full[i % UNITS]));
      }
      __syncwarp();
      if (u.r.b < 0) break;
    }
  } else if (warp == 1) {
    // =========================== V: a buffer is free again once P V of the tile NB before has completed ==================
    const uint32_t full_lead = map_rank(smem_u32(&v_full[0]), 0);
    const int nb = np * (L::VN / 128 / cb), blk = lane / nb, pc = lane % np, ch = ((lane % nb) / np) * cb;   // copies of a block; block of this lane
    uint32_t ph_own = 0;
    int n = 0, i = 0;
    Ring<NB> rg;
    for (Unit u = unit(0); u.r.b >= 0; u = unit(++i)) {
      for (int t = 0; t < u.T; ++t, ++n, rg.next()) {
        const int key0 = (u.t0 + t) * KB, rem = u.r.kv - key0;                        // rows past the cached tokens: rem .. of the tile
        // (rows up to the end of the piece that they begin in; later pieces are zeros)
        const int clear_to = (rem + (1 << piece_shift) - 1) >> piece_shift << piece_shift;
        const bool fetch = DH >= 128 || half == 0, clear = fetch && rem > 0 && rem < KB && clear_to > rem;
        const int row = fetch && lane < 2 * nb ? row_of(u.r, key0 + blk * 64 + (pc << piece_shift)) : 0;
        const int bf = rg.at;
        const uint32_t dst = Vs + (uint32_t)bf * L::VTILE;
        uint32_t bar = smem_u32(&v_full[bf]);
        if (lane == 0) {
          if (n >= NB) wait(smem_u32(&pv_done[bf]), rg.parity ^ 1u, wl);
          if (clear) mbar_expect_tx(smem_u32(&v_own), (uint32_t)L::VTILE);
          else if (half == 0) mbar_expect_tx(bar, (DH < 128 ? 1 : 2) * (uint32_t)L::VTILE);
          else remote_arrive(full_lead + (uint32_t)bf * 8u);
        }
        __syncwarp();
        if (n == 0) first_copies();
        bar = clear ? smem_u32(&v_own) : bar & LEADER_MASK;
        if (fetch && lane < 2 * nb)
          copy4d(dst + (uint32_t)blk * L::PIECE + (uint32_t)ch * L::KBLOCK + (uint32_t)pc * piece_bytes, &tmkv, row, u.hk * (DH / 64) + half * (DH / 128) + ch,
                 a.plane + 1, bar);
        if (clear) {
          wait_warp(bar, ph_own, wl);
          ph_own ^= 1u;
          for (int i = lane; i < (clear_to - rem) * (L::VN / 16); i += 32) {           // (a row: 8 x 16 bytes in each of VN / 128 blocks)
            const int r = rem + i / (L::VN / 16), c = i % (L::VN / 16);
            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(dst + (uint32_t)((r >> 6) * L::PIECE + (c >> 3) * L::KBLOCK + (r & 63) * 128 + (c & 7) * 16)), "r"(0u) : "memory");
          }
          fence_async_smem();                    // generic-proxy writes, read next by the tensor cores
          __syncwarp();
          if (lane == 0) remote_arrive_stores(full_lead + (uint32_t)bf * 8u);
        }
      }
    }
    __syncwarp();
  } else if (warp == 3) {
    // =========================== MMA issuer (leader CTA): S(0) .. S(NB - 1), then P(n) V(n), S(n + NB), across the units ==========
    // The products wait for one another through what stands between their MMAs: S(n + NB) follows P(n) V(n), whose P is in its buffer, in the
    // pipe's order.  So the loop is short: plain waits in a fixed order, one election, four MMAs a statement.  (Whichever of the two had its
    // operands first, an election per MMA: 600 to 900 clocks from the last MMA of a product to the first of the next, beside two busy warps of
    // the scheduler, 3400 per tile.  Two warps, one per product: 2770, as S(n + NB) then waits for the completion of P(n) V(n).)
    if (half == 0) {
      const uint32_t elected = elect_one() ? 1u : 0u;
      // ahead: logits issued whose P V has not been; left: tiles of the unit whose logits are to come.  The logits' unit is this one or the next.
      int ahead = 0, left = 0, i = 0;
      uint32_t par_q = 1, par_o = 1;
      Ring<NB> rs, rp;
      const uint32_t k_bar = smem_u32(&k_full[0]), s_bar = smem_u32(&s_full[0]), v_bar = smem_u32(&v_full[0]), p_bar = smem_u32(&p_full[0][0]), d_bar = smem_u32(&pv_done[0]);
      const uint64_t dq = make_desc(Qs), dk = make_desc(Ks), dv = make_desc_mn(Vs, L::KBLOCK, 1024);
      Unit u = unit(0), nx = u;
      bool next_begun = true;                                     // (the logits' unit is nx)
      if (u.r.b >= 0) {
        left = u.T, par_q ^= 1u;
        wait_warp(smem_u32(&q_full), par_q, wc);
        nx = unit(1), next_begun = false;
      }
      for (; u.r.b >= 0; ++i, par_o ^= 1u) {
        const int ends = u.r.kv < (u.t0 + u.T) * KB ? u.T - 1 : -1;       // the tile in which the cached tokens end: rows of it were cleared by a warp of each CTA
        for (int t = 0; t < u.T; ++t) {
          // Logits as far ahead as there are buffers; those of the next unit only once its queries are there, or nothing else is left
          do {
            if (left == 0) {
              if (next_begun || nx.r.b < 0 || !(ahead == 0 || __all_sync(0xffffffffu, mbar_test(smem_u32(&q_full), par_q ^ 1u)))) break;
              left = nx.T, par_q ^= 1u, next_begun = true;
              wait_warp(smem_u32(&q_full), par_q, wc);
            }
            wait_warp(k_bar + 8u * rs.at, rs.parity, wc);
            tc_fence_after();
            const uint64_t db = dk + (uint64_t)((uint32_t)rs.at * (L::KTILE >> 4));      // (a 64-channel block further: 128 x 128 and 64 x 128 bytes)
#pragma unroll
            for (int c = 0; c < DH / 64; ++c)
              umma2_ss_x4(tmem_s + (uint32_t)rs.at * KB, dq + (uint64_t)(c * ((128 * 128) >> 4)), db + (uint64_t)(c * (L::KBLOCK >> 4)), IDESC_S, c == 0 ? 1u : 0u, elected);
            if (elected) {
              umma2_commit(s_bar + 8u * rs.at);
              if (left == 1) umma2_commit(smem_u32(&q_free));
            }
            rs.next(), ++ahead, --left;
          } while (ahead < NB);
          wait_warp(v_bar + 8u * rp.at, rp.parity, wc);
          if (t == ends) pair_acquire(v_bar + 8u * rp.at, rp.parity);
          if (t == 0 && i > 0) wait_warp(smem_u32(&o_free), par_o, wc);
#pragma unroll
          for (int kh = 0; kh < 2; ++kh) {
            wait_warp(p_bar + 16u * rp.at + 8u * kh, rp.parity, wc);
            tc_fence_after();
            // A = P of this tile: bf16 pairs in the first 64 columns of its S buffer
            umma2_ts_x4(tmem_o, tmem_s + (uint32_t)rp.at * KB + (uint32_t)kh * 32, dv + (uint64_t)((uint32_t)rp.at * (L::VTILE >> 4) + kh * (L::PIECE >> 4)), IDESC_PV,
                        t == 0 && kh == 0 ? 1u : 0u, elected);
          }
          if (elected) umma2_commit(d_bar + 8u * rp.at);
          rp.next(), --ahead;
        }
        // (with units of one tile the logits of the next one may be all issued: then on to the one behind it)
        u = nx;
        if (u.r.b >= 0) {
          if (!next_begun) {
            left = u.T, par_q ^= 1u;
            wait_warp(smem_u32(&q_full), par_q, wc);
          }
          nx = unit(i + 2), next_begun = false;
        }
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    // =========================== softmax / correction / output ==============================================================
    const int g = (warp - 4) >> 2;            // part of a row's columns
    const int q = warp & 3;
    const int row = q * 32 + lane;            // accumulator row = tensor-memory lane
    const int row_tok = row / G;              // token of the CTA's TOK (rows past TOK * G: none)
    const uint32_t lane_addr = (uint32_t)(q * 32) << 16;
    const uint32_t pfull0 = map_rank(smem_u32(&p_full[0][g >> 1]), 0), ofree0 = map_rank(smem_u32(&o_free), 0);
    const uint32_t ostage = Qs + L::QTILE + (uint32_t)(warp - 4) * L::STG;
    const int c0 = g * (DH / 4);              // first of this warp's output channels
    int out_off[2];                           // where this lane stores of a unit's rows (lane / 2 + 16 x of the warp's 32)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = q * 32 + (lane >> 1) + 16 * x, rt = r / G;
      out_off[x] = (rt * a.hq + r - rt * G) * DH + c0 + (lane & 1) * 8;
    }
    bool odd = false;
    int n = 0, i = 0;
    Ring<NB> rg;
    uint32_t last_bar = 0, last_par = 0;      // of the tile before: its P V complete
    for (Unit me = unit(0); me.r.b >= 0; me = unit(++i)) {
      const int tok = me.tok0 + half * TOK + row_tok;
      const bool live = row < TOK * G && tok < me.r.n;
      // (rows of no token count as seeing all: masked, they would keep their warps in the masked form of every tile)
      const int lim = live ? me.r.limit(tok, a.causal) - me.t0 * KB - g * 32 : 0x40000000;
      float m = -INFINITY, l = 0.f;           // running maximum (log2 units) and sum (of this thread's columns)
      for (int t = 0; t < me.T; ++t, ++n, rg.next()) {
        wait_warp(smem_u32(&s_full[rg.at]), rg.parity, wc);
        tc_fence_after();
        softmax_tile<DH>(m, l, xch[n & 1], tmem_s + (uint32_t)rg.at * KB + lane_addr, tmem_o + lane_addr, g, q, row, live ? lim - t * KB : KB, live, a.scale_log2,
                         [&] { wait_warp(last_bar, last_par, wc); });
        if (lane == 0) remote_arrive(pfull0 + (uint32_t)rg.at * 16u);
        last_bar = smem_u32(&pv_done[rg.at]), last_par = rg.parity;
      }
      // ---- output: O / l -> bf16, 16 columns at a time through a staging block of the warp, out in whole sectors; or the accumulator
      // of a key range as it is.  A rolled loop: run once per unit, its code comes from far at about 11 clocks an instruction.
      xsum[i & 1][g][row] = l;
      rows_sync(q);
      const float sum = (xsum[i & 1][0][row] + xsum[i & 1][1][row]) + (xsum[i & 1][2][row] + xsum[i & 1][3][row]);
      const bool sees = live && me.r.limit(tok, a.causal) > 0;
      const float inv = paged_inv(sum, sees);
      wait_warp(last_bar, last_par, wc);
      tc_fence_after();
      const bool okf = !skip && !*reinterpret_cast<volatile int*>(&abort_flag);
      const int first_tok = me.r.lo + me.tok0 + half * TOK, n_rows = okf ? min(TOK, me.r.n - me.tok0 - half * TOK) * G : 0;
      const bool whole = me.ranges == 1;
      const size_t slot = ((size_t)me.range * a.pb.tokens + first_tok + row_tok) * a.hq + me.hk * G + (row - row_tok * G);
      if (g == 0 && a.ranges > 1 && row < n_rows) a.part_ml[slot] = make_float4(m, sum, (float)me.ranges, sees ? 1.f : 0.f);
      __nv_bfloat16* ob = (__nv_bfloat16*)a.out + ((size_t)first_tok * a.hq + me.hk * G) * DH;
      float fin = 0.f;
#pragma unroll 1
      for (int c = 0; c < DH / 4; c += 16, ob += 16) {
        float o[16];
        tmem_ld16(tmem_o + lane_addr + (uint32_t)(c0 + c), o);
        if (c + 16 == DH / 4) {               // the accumulator may be overwritten
          tc_fence_before();
          __syncwarp();
          if (lane == 0) remote_arrive(ofree0);
        }
        if (!whole) {
          if (row < n_rows) {
            float* p = a.part_o + slot * DH + c0 + c;
#pragma unroll
            for (int e = 0; e < 16; e += 8)        // (whole sectors)
              asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p + e), "f"(o[e]), "f"(o[e + 1]), "f"(o[e + 2]), "f"(o[e + 3]), "f"(o[e + 4]),
                           "f"(o[e + 5]), "f"(o[e + 6]), "f"(o[e + 7])
                           : "memory");
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) fin = fmaf(o[e], 0.f, fin);
          continue;
        }
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          fin = fmaf(o[2 * e], 0.f, fin), fin = fmaf(o[2 * e + 1], 0.f, fin);        // (NaN of an infinity or a NaN)
          w[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(ostage + (uint32_t)(lane * 32 + ((e ^ ((lane >> 2) & 1)) << 4))), "r"(w[4 * e]), "r"(w[4 * e + 1]),
                       "r"(w[4 * e + 2]), "r"(w[4 * e + 3])
                       : "memory");
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int rr = (lane >> 1) + 16 * x;
          uint4 v;
          asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                       : "r"(ostage + (uint32_t)(rr * 32 + (((lane & 1) ^ ((rr >> 2) & 1)) << 4))) : "memory");
          if (q * 32 + rr < n_rows) *reinterpret_cast<uint4*>(ob + out_off[x]) = v;
        }
        __syncwarp();
      }
      odd |= row < n_rows && !(fin == 0.f);
    }
    // ---- rows that are not finite although the values that they see may be: those of them with an infinity or a NaN among the keys of
    // their tiles that they do not see once more, key by key (channel by channel right otherwise: an infinite value is of one channel)
    if (a.causal) {
      __threadfence();
      rows_sync(q);                           // (maxima beside a range's result: written by another warp of the quarter)
    }
    // (the warp as one: another warp may raise the flag under it)
    if (a.causal && __any_sync(0xffffffffu, odd) && !__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&abort_flag) != 0)) {
      int at = s_list[2];
      for (Unit u = next_unit(at, s_list[0], s_list[1]); u.r.b >= 0; u = next_unit(at, s_list[0], s_list[1])) {
        const int n_rows = min(TOK, u.r.n - u.tok0 - half * TOK) * G, end = min((u.t0 + u.T) * KB, u.r.kv);
        for (int rr = q * 32; rr < min(n_rows, q * 32 + 32); ++rr) {
          const int rt = rr / G, tok = u.r.lo + u.tok0 + half * TOK + rt, head = u.hk * G + rr - rt * G;
          const int lim = u.r.limit(u.tok0 + half * TOK + rt, 1);
          const size_t slot = ((size_t)u.range * a.pb.tokens + tok) * a.hq + head;
          __nv_bfloat16* ob = (__nv_bfloat16*)a.out + ((size_t)tok * a.hq + head) * DH + c0;
          float* of = a.part_o + slot * DH + c0;
          bool bad_row = false;
          for (int e = lane; e < DH / 4; e += 32) bad_row |= !(fabsf(u.ranges == 1 ? __bfloat162float(ob[e]) : of[e]) < INFINITY);
          if (!__any_sync(0xffffffffu, bad_row)) continue;
          if (!paged_hidden_odd<DH / 32, __nv_bfloat16>(a, u.r.b, u.hk, DH, 0, max(u.t0 * KB, lim), end)) continue;
          float o[DH / 32], M, sum;
          paged_row_alone<DH>(a, u.r.b, (const __nv_bfloat16*)a.q + tok * a.q_stride + (long long)head * DH, u.hk, u.t0 * KB, min(end, lim), o, M, sum);
          // (a key range's result is relative to the maximum that stands beside it)
          const float w = u.ranges == 1 ? paged_inv(sum, lim > 0) : M == -INFINITY ? 0.f : exp2f(M - a.part_ml[slot].x);
#pragma unroll
          for (int e = 0; e < DH / 32; ++e) {
            const int c = lane * (DH / 32) + e - c0;
            if (c < 0 || c >= DH / 4) continue;
            if (u.ranges == 1) ob[c] = __float2bfloat16_rn(o[e] * w);
            else of[c] = o[e] * w;
          }
        }
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  // Neither CTA leaves (or gives its tensor memory back) while the other still works: the leader's MMAs read both CTAs'
  // shared memory and write both tensor memories.
  cluster_arrive_relaxed();
  cluster_wait();
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc2(tmem_base, 512);
  }
}

// query rows: copies of 64 channels of `group` heads of 128 / group tokens
bool query_map(CUtensorMap* m, const PagedAttn& a, int dh) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return false;
  const cuuint64_t dims[4] = {64, (cuuint64_t)a.hq, (cuuint64_t)a.pb.tokens, (cuuint64_t)dh / 64};
  const cuuint64_t strides[3] = {(cuuint64_t)dh * 2, (cuuint64_t)a.q_stride * 2, 128};
  const cuuint32_t box[4] = {64, (cuuint32_t)a.group, (cuuint32_t)(128 / a.group), 1}, es[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH>
cudaError_t setup_one() {
  static PerDeviceOnce once;
  if (!once.needed()) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(k_paged_pair<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PpLayout<DH>::SMEM);
  if (e == cudaSuccess) once.done();
  return e;
}
template <int DH>
int resident_one() {
  if (setup_one<DH>() != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(1024), cfg.blockDim = dim3(PP_THREADS), cfg.dynamicSmemBytes = PpLayout<DH>::SMEM;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
  cfg.attrs = at, cfg.numAttrs = 1;
  int n = 0;
  return cudaOccupancyMaxActiveClusters(&n, k_paged_pair<DH>, &cfg) == cudaSuccess ? n : 0;
}

template <int DH>
cudaError_t launch_one(const PagedAttn& a, const phyai_paged_cache_t* cache, long long items, cudaStream_t st) {
  cudaError_t e = setup_one<DH>();
  if (e != cudaSuccess) return e;
  const int pairs = paged_pair_resident(DH);
  if (items < 1 || pairs < 1) return cudaErrorInvalidConfiguration;
  const int piece_shift = a.pb.page_shift < 6 ? a.pb.page_shift : 6;
  CUtensorMap tq, tkv;
  if (!query_map(&tq, a, DH) || !paged_pool_map(&tkv, cache, 1u << piece_shift, piece_shift == 6 ? PpLayout<DH>::VN / 128 : 1)) return cudaErrorInvalidValue;
  const unsigned grid = 2u * (unsigned)(items < pairs ? items : pairs);
  return launch_pdl(k_paged_pair<DH>, dim3(grid), dim3(PP_THREADS), PpLayout<DH>::SMEM, st, a, tq, tkv, piece_shift);
}

}  // namespace

bool paged_pair_supported(int dh, int group) { return (dh == 64 || dh == 128 || dh == 256) && group <= 128 && paged_pair_resident(dh) > 0; }
int paged_pair_tokens(int group) { return 2 * (128 / group); }

int paged_pair_resident(int dh) {
  static PerDeviceCount resident[3];
  return dh == 256 ? resident[2].get(resident_one<256>) : dh == 128 ? resident[1].get(resident_one<128>) : resident[0].get(resident_one<64>);
}

cudaError_t launch_paged_pair(const PagedAttn& a, const phyai_paged_cache_t* cache, long long items, cudaStream_t st) {
  return cache->head_dim == 256 ? launch_one<256>(a, cache, items, st) : cache->head_dim == 128 ? launch_one<128>(a, cache, items, st) : launch_one<64>(a, cache, items, st);
}

}  // namespace phyai
