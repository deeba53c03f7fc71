// What writes and drains the paged cache, and the heads' norm and rotation on their own:
//   phyai_norm_rope_heads   q, k rows -> normed, rotated rows
//   phyai_append_paged_kv   the same for k, written into the pages with v; q rows in the same pass when given
//   phyai_pack_paged_kv     pages -> the ragged prefix cache that the denoising loop reads
//
// A head x of dh channels becomes  y = x * rsqrt(mean(x^2) + eps) * (1 + gain)  and then, for j < dh / 2,
//   (y_j, y_{j + dh/2}) -> (y_j cos - y_{j + dh/2} sin, y_{j + dh/2} cos + y_j sin)  with the table's row of its position.
// Everything is read once and written once, so memory bounds it: a lane takes 16 bytes of a head's channels and their rotary partners, so
// that only the sum of squares crosses lanes (with 8 channels a lane and the partners by shuffles, shuffles and table loads bounded it).  The
// channels are pairs, a warp's next to one another: a pair's table entry is 16 bytes, so that a load of the table or the gains takes as few passes of
// the L1 as it can (with 8 channels in a row, one load of 16 bytes, a lane's entries are 64 bytes apart: 17.1 for 15.0 us).  The arithmetic is
// fp32 with one rounding at the store.
// Measured: 7744 tokens of 9 heads of 256 (pi0), bf16, rows from memory: 16.5 us, 4.4 TB/s (14.6 where the 72 MB lie in the L2, as in the figures of variants
// here); 6272 tokens with the append (k, v into pages) 17.0 (14.5).  Nothing is full (58 % of the issue slots, 43 % of the L1): a warp loads two slots, computes,
// stores and only then loads again.  64 tokens: 2 - 3 us, the chain lengths -> page -> table -> store.  Packing 231 MB: 39.2 us, 5.9 TB/s of 6.55
// that a copy reaches.
#include <atomic>
#include <cstdio>

#include "../../include/phyai.h"
#include "paged.cuh"

namespace phyai {

thread_local char g_paged_err[256] = "";

namespace {

// A lane's channels of half a head, as stored: 16 bytes, in pairs `apart` channels from one another.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  static constexpr int N = 4;
  float2 a[2];
  __device__ __forceinline__ void load(const float* p, int apart) {
#pragma unroll
    for (int j = 0; j < 2; ++j) a[j] = *reinterpret_cast<const float2*>(p + j * apart);
  }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = a[0].x, v[1] = a[0].y, v[2] = a[1].x, v[3] = a[1].y; }
};
template <>
struct Raw<__nv_bfloat16> {
  static constexpr int N = 8;
  uint32_t a[4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int apart) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = *reinterpret_cast<const uint32_t*>(p + j * apart);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(a[i] << 16), v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
  }
};
template <int N>
__device__ __forceinline__ void store_channels(float* p, const float (&x)[N], int apart) {
#pragma unroll
  for (int i = 0; i < N; i += 2) *reinterpret_cast<float2*>(p + i / 2 * apart) = make_float2(x[i], x[i + 1]);
}
template <int N>
__device__ __forceinline__ void store_channels(__nv_bfloat16* p, const float (&x)[N], int apart) {
#pragma unroll
  for (int i = 0; i < N; i += 2) *reinterpret_cast<__nv_bfloat162*>(p + i / 2 * apart) = __floats2bfloat162_rn(x[i], x[i + 1]);
}

struct HeadsArgs {
  const void *q, *k, *v;                 // token rows, heads contiguous in a row; q or v may be null
  long long q_stride, k_stride, v_stride;   // elements
  int hq, hkv, tokens;
  const int* positions;                  // [tokens] or null (append: the token's place in the cache)
  const float* rope;                     // [n_positions][dh / 2][2] or null
  int n_positions;
  const float *q_gain, *k_gain;          // [dh] or null: no norm
  float eps;
  void *q_out, *k_out;                   // contiguous rows (k_out: norm_rope_heads)
  void *k_plane, *v_plane;               // append: the layer's planes
  PagedBatch pb;
  int* status;
};

constexpr int HT = 256, HB = 4;          // threads of a block, blocks of an SM

// A lane takes C channels and their rotary partners of a head, a warp 64 C / dh heads of a token at a time (a slot); slots run over the tokens, a
// warp takes U in a row and issues all their loads before it uses the first.  Two slots and four blocks: 15.0 us for the above; one slot 15.0 (append
// 14.8 for 14.5), three 18.8, three blocks 15.7, five 17 and more (spills); the loads of the next slots under these: 18.7 (registers).
template <int DH, typename IN, typename OUT, bool APPEND, int U>
__global__ void __launch_bounds__(HT, HB) k_heads(const HeadsArgs a) {
  constexpr int C = Raw<IN>::N, HALF = DH / 2, LANES = HALF / C, HPS = 32 / LANES, APART = LANES * 2;           // lanes per head, heads per slot
  __shared__ int s_cu[APPEND ? PAGED_MAX_BATCH + 1 : 1], s_kv[APPEND ? PAGED_MAX_BATCH : 1], s_skip;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LANES, c = (lane % LANES) * 2;
  const int hq = a.q ? a.hq : 0, H = hq + a.hkv + (a.v ? a.hkv : 0), slots = (H + HPS - 1) / HPS;
  const int step = (int)gridDim.x * (HT / 32) * U, step_tok = step / slots, step_slot = step - step_tok * slots;
  pdl_launch_dependents();
  pdl_wait();
  if constexpr (APPEND) {
    if (threadIdx.x == 0) s_skip = paged_stopped(a.status, a.pb);
    bool bad = false;
    for (int i = threadIdx.x; i < a.pb.batch; i += HT) {
      const int lo = a.pb.cu[i], hi = a.pb.cu[i + 1], kv = a.pb.kv_lens[i];
      bad |= paged_entry_bad(a.pb, i, lo, hi, kv, true);
      s_cu[i] = lo, s_kv[i] = kv;
      if (i + 1 == a.pb.batch) s_cu[i + 1] = hi;
    }
    bad = __syncthreads_or(bad);
    if (bad) {
      if (threadIdx.x == 0) paged_raise(a.status, a.pb);
      return;
    }
    if (s_skip) return;
  }

  const int s0 = ((int)blockIdx.x * (HT / 32) + warp) * U;
  for (int tok0 = s0 / slots, slot0 = s0 % slots; tok0 < a.tokens;) {
    Raw<IN> lo[U], hi[U];
    {
      int tok = tok0, slot = slot0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = slot * HPS + sub;
        if (h < H && tok < a.tokens) {
          const IN* p = h < hq ? (const IN*)a.q + tok * a.q_stride + h * DH
                               : h < hq + a.hkv ? (const IN*)a.k + tok * a.k_stride + (h - hq) * DH : (const IN*)a.v + tok * a.v_stride + (h - hq - a.hkv) * DH;
          lo[u].load(p + c, APART), hi[u].load(p + c + HALF, APART);
        } else {
          lo[u] = hi[u] = Raw<IN>{};
        }
        if (++slot == slots) slot = 0, ++tok;
      }
    }
    float cs[C], sn[C];
    long long row = -1;
    bool ok = false;
    int tok = tok0, slot = slot0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (tok >= a.tokens) break;
      if (u == 0 || slot == 0) {                                 // ---- another token: where it is
        int pos = 0;
        ok = true;
        if constexpr (APPEND) {
          int b = 0;                                             // requests that end at or before it
          for (int i0 = 0; i0 < a.pb.batch; i0 += 32) b += __popc(__ballot_sync(0xffffffffu, i0 + lane < a.pb.batch && s_cu[min(i0 + lane, a.pb.batch - 1) + 1] <= tok));
          ok = tok >= s_cu[0] && b < a.pb.batch;                 // (else a row of no request)
          if (ok) {
            const int place = s_kv[b] - (s_cu[b + 1] - tok);
            row = paged_row(a.pb, b, place);
            pos = a.positions ? a.positions[tok] : place;
            if (row < 0 || (a.rope && (unsigned)pos >= (unsigned)a.n_positions)) {
              if (lane == 0) paged_bad_entry(a.status, a.pb);
              ok = false;                                        // (nothing of this token is written)
            }
          }
        } else if (a.rope) {
          pos = a.positions[tok];
          ok = (unsigned)pos < (unsigned)a.n_positions;
          if (!ok && lane == 0) paged_raise(a.status, a.pb);
        }
        if (ok && a.rope) {
          const float* t = a.rope + ((size_t)pos * HALF + c) * 2;
#pragma unroll
          for (int i = 0; i < C; i += 2) {
            const float4 w = __ldg(reinterpret_cast<const float4*>(t + i * APART));
            cs[i] = w.x, sn[i] = w.y, cs[i + 1] = w.z, sn[i + 1] = w.w;
          }
        }
      }
      const int h = slot * HPS + sub, kind = h < hq ? 0 : h < hq + a.hkv ? 1 : h < H ? 2 : 3;
      float x[C], y[C];
      lo[u].get(x), hi[u].get(y);
      const float* gain = kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr;
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < C; ++i) ss = fmaf(x[i], x[i], ss), ss = fmaf(y[i], y[i], ss);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (gain) {
        const float r = rsqrtf(ss * (1.0f / DH) + a.eps);
#pragma unroll
        for (int i = 0; i < C; i += 2) {
          const float* at = gain + c + i / 2 * APART;
          const float2 g = __ldg(reinterpret_cast<const float2*>(at)), f = __ldg(reinterpret_cast<const float2*>(at + HALF));
          x[i] *= fmaf(r, g.x, r), x[i + 1] *= fmaf(r, g.y, r);
          y[i] *= fmaf(r, f.x, r), y[i + 1] *= fmaf(r, f.y, r);
        }
      }
      if (a.rope && kind < 2) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const float t = x[i];
          x[i] = fmaf(-y[i], sn[i], t * cs[i]);
          y[i] = fmaf(t, sn[i], y[i] * cs[i]);
        }
      }
      if (!APPEND && !ok) {                                      // (whoever does not look at the word sees it)
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = y[i] = NAN;
      }
      if ((ok || !APPEND) && kind < 3) {
        OUT* p = kind == 0 ? (OUT*)a.q_out + ((size_t)tok * a.hq + h) * DH
                 : APPEND  ? (OUT*)(kind == 1 ? a.k_plane : a.v_plane) + ((size_t)row * a.hkv + (kind == 1 ? h - hq : h - hq - a.hkv)) * DH
                           : (OUT*)a.k_out + ((size_t)tok * a.hkv + h - hq) * DH;
        store_channels(p + c, x, APART), store_channels(p + c + HALF, y, APART);
      }
      if (++slot == slots) slot = 0, ++tok;
    }
    tok0 += step_tok, slot0 += step_slot;
    if (slot0 >= slots) slot0 -= slots, ++tok0;
  }
}

constexpr int NOTES = 4096;
__device__ unsigned g_raised_by[NOTES];

}  // namespace

cudaError_t paged_call(const int32_t* status_word, PagedBatch* p) {
  static std::atomic<unsigned> calls{0};
  static std::atomic<unsigned*> notes[64] = {};
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  unsigned* at = dev < 64 ? notes[dev].load(std::memory_order_acquire) : nullptr;
  if (!at) {
    e = cudaGetSymbolAddress(reinterpret_cast<void**>(&at), g_raised_by);
    if (e != cudaSuccess) return e;
    if (dev < 64) notes[dev].store(at, std::memory_order_release);
  }
  // (words are often 512 bytes apart: all bits of the address count)
  p->raised_by = at + ((reinterpret_cast<uintptr_t>(status_word) >> 2) * 0x9E3779B97F4A7C15ull >> 52);
  do p->call = calls.fetch_add(1, std::memory_order_relaxed) + 1;
  while (p->call == 0);                                          // (0: no call)
  return cudaSuccess;
}

int paged_sm_count() {
  static PerDeviceCount n;
  return n.get([] {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return v;
  });
}

namespace {

template <int DH, typename IN, typename OUT, bool APPEND>
cudaError_t launch_heads(const HeadsArgs& a, cudaStream_t st) {
  constexpr int HPS = 64 * Raw<IN>::N / DH, U = 2;
  const int H = (a.q ? a.hq : 0) + a.hkv + (a.v ? a.hkv : 0), slots = (H + HPS - 1) / HPS, n_sm = paged_sm_count();
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const long long n = (long long)a.tokens * slots;
  if (n > 0x7f000000ll) return cudaErrorInvalidValue;
  // Few tokens: a warp per slot, all of them at a time; many: U slots a warp.
  if (n <= (long long)n_sm * 16)
    return launch_pdl(k_heads<DH, IN, OUT, APPEND, 1>, dim3((unsigned)((n + HT / 32 - 1) / (HT / 32))), dim3(HT), 0, st, a);
  const long long blocks = (n + U * (HT / 32) - 1) / (U * (HT / 32)), most = (long long)n_sm * HB;
  return launch_pdl(k_heads<DH, IN, OUT, APPEND, U>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(HT), 0, st, a);
}
template <bool APPEND>
cudaError_t dispatch_heads(int dh, uint32_t in, uint32_t out, const HeadsArgs& a, cudaStream_t st) {
  using bf = __nv_bfloat16;
#define PHYAI_HEADS(DH)                                                                         \
  if (dh == DH) {                                                                               \
    if (in == PHYAI_BF16) return launch_heads<DH, bf, bf, APPEND>(a, st);                       \
    if (out == PHYAI_BF16) return launch_heads<DH, float, bf, APPEND>(a, st);                   \
    return launch_heads<DH, float, float, APPEND>(a, st);                                       \
  }
  PHYAI_HEADS(64)
  PHYAI_HEADS(128)
  PHYAI_HEADS(256)
#undef PHYAI_HEADS
  return cudaErrorInvalidValue;
}

// Pages -> packed rows.  Blocks move 16 KB of one plane (grid.y) and request (grid.z) at a time, four 16-byte loads a thread, every gridDim.x-th
// chunk; every block adds up the lengths before its request itself, the loads of its first chunk on their way.
constexpr int PP_T = 256, PP_U = 4, PP_CHUNK = PP_T * PP_U;
__global__ void __launch_bounds__(PP_T) k_pack_pages(const uint4* pages, uint4* dst, int* cu, int* status, const PagedBatch p, long long kv_tokens,
                                                     int row_chunks) {
  __shared__ long long s_part[2][PP_T / 32];
  __shared__ int s_skip;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.z;
  pdl_launch_dependents();
  pdl_wait();
  if (tid == 0) s_skip = paged_stopped(status, p);
  const int my_len = p.kv_lens[b];
  const bool first = blockIdx.x == 0 && blockIdx.y == 0;
  const int page_chunks = row_chunks << p.page_shift;
  const bool in_range = my_len >= 0 && (long long)my_len <= ((long long)p.max_pages << p.page_shift);
  const int n = in_range ? my_len * row_chunks : 0;
  if ((int)blockIdx.x * PP_CHUNK >= n && !first) return;
  const size_t plane_chunks = ((size_t)p.n_pages << p.page_shift) * row_chunks;
  const uint4* src = pages + (size_t)blockIdx.y * plane_chunks;
  uint4 x[PP_U];
  bool have[PP_U], bad_page = false;
  auto load = [&](long long i0) {
#pragma unroll
    for (int u = 0; u < PP_U; ++u) {
      const long long i = i0 + u * PP_T;
      have[u] = false;
      if (i < n) {
        const int pg = (int)i / page_chunks, page = p.table[(size_t)b * p.max_pages + pg];
        have[u] = (unsigned)page < (unsigned)p.n_pages;
        bad_page |= !have[u];
        if (have[u]) x[u] = __ldcs(src + (size_t)page * page_chunks + ((int)i - pg * page_chunks));
      }
    }
  };
  long long i0 = (long long)blockIdx.x * PP_CHUNK + tid;
  load(i0);
  // ---- rows before this request, all rows
  long long before = 0, total = 0;
  bool bad = false;
  for (int i = tid; i < p.batch; i += PP_T) {
    const int len = p.kv_lens[i];
    bad |= len < 0 || (long long)len > ((long long)p.max_pages << p.page_shift);
    total += max(len, 0);
    if (i < b) before += max(len, 0);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o), total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) s_part[0][warp] = before, s_part[1][warp] = total;
  bad = __syncthreads_or(bad);
  before = total = 0;
#pragma unroll
  for (int w = 0; w < PP_T / 32; ++w) before += s_part[0][w], total += s_part[1][w];
  bad |= total > kv_tokens;
  if (s_skip) return;
  if (bad) {
    if (first && tid == 0) paged_raise(status, p);
    return;
  }
  if (first && tid == 0) {
    if (b == 0) cu[0] = 0;
    cu[b + 1] = (int)(before + my_len);                     // (at most kv_tokens < 2^31)
  }
  uint4* const o = dst + ((size_t)blockIdx.y * kv_tokens + before) * row_chunks;
  for (;;) {
#pragma unroll
    for (int u = 0; u < PP_U; ++u)
      if (have[u]) o[i0 + u * PP_T] = x[u];
    i0 += (long long)gridDim.x * PP_CHUNK;
    if (i0 - tid >= n) break;
    load(i0);
  }
  if (bad_page) paged_bad_entry(status, p);
}

phyai_status_t bad_arg(const char* m) {
  snprintf(g_paged_err, sizeof(g_paged_err), "%s", m);
  return PHYAI_ERR_INVALID_ARG;
}
phyai_status_t launch_result(cudaError_t e) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e == cudaSuccess) return PHYAI_OK;
  snprintf(g_paged_err, sizeof(g_paged_err), "kernel launch failed: %s", cudaGetErrorString(e));
  return PHYAI_ERR_CUDA;
}
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

phyai_status_t check_heads(const phyai_heads_desc_t* d, uint32_t tokens, const void* q, uint64_t q_stride, const void* k, uint64_t k_stride,
                           const float* rope, uint64_t n_positions, const float* q_gain, const float* k_gain, const void* q_out,
                           const int32_t* status_word) {
  if (!d || d->struct_size != sizeof(phyai_heads_desc_t)) return bad_arg("desc is NULL or has a wrong struct_size");
  if (!d->n_kv_heads || (q && !d->n_q_heads)) return bad_arg("a head count in desc is zero");
  if (d->n_q_heads > 65535u || d->n_kv_heads > 65535u || tokens > 0x7fffffffu) return bad_arg("too many heads or tokens");
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) {
    snprintf(g_paged_err, sizeof(g_paged_err), "head_dim must be 64, 128 or 256");
    return PHYAI_ERR_UNSUPPORTED;
  }
  const bool types = (d->in_dtype == PHYAI_BF16 && d->out_dtype == PHYAI_BF16) || (d->in_dtype == PHYAI_F32 && (d->out_dtype == PHYAI_BF16 || d->out_dtype == PHYAI_F32));
  if (!types) {
    snprintf(g_paged_err, sizeof(g_paged_err), "types must be bfloat16 -> bfloat16, float32 -> bfloat16 or float32 -> float32");
    return PHYAI_ERR_UNSUPPORTED;
  }
  if (!status_word || (tokens && (!k || (q && !q_out)))) return bad_arg("a pointer argument is NULL");
  const uint64_t es = d->in_dtype == PHYAI_F32 ? 4 : 2;
  if ((q && q_stride < (uint64_t)d->n_q_heads * d->head_dim) || k_stride < (uint64_t)d->n_kv_heads * d->head_dim ||
      q_stride > (1ull << 40) || k_stride > (1ull << 40))
    return bad_arg("a row stride is smaller than the row's heads, or too large");
  if (!aligned16(q) || !aligned16(k) || !aligned16(rope) || !aligned16(q_gain) || !aligned16(k_gain) || !aligned16(q_out) ||
      (q && (q_stride * es) % 16) || (k_stride * es) % 16)
    return bad_arg("pointers and row strides must be multiples of 16 bytes");
  if (!aligned4(status_word)) return bad_arg("status_word must be 4-byte aligned");
  if (rope && (n_positions == 0 || n_positions > 0x7fffffffull)) return bad_arg("n_positions out of range");
  return PHYAI_OK;
}

HeadsArgs heads_args(const phyai_heads_desc_t* d, uint32_t tokens, const void* q, uint64_t q_stride, const void* k, uint64_t k_stride,
                     const int32_t* positions, const float* rope, uint64_t n_positions, const float* q_gain, const float* k_gain, void* q_out,
                     int32_t* status_word) {
  HeadsArgs a{};
  a.q = q, a.k = k, a.q_stride = (long long)q_stride, a.k_stride = (long long)k_stride, a.hq = (int)d->n_q_heads, a.hkv = (int)d->n_kv_heads;
  a.tokens = (int)tokens, a.positions = positions, a.rope = rope, a.n_positions = (int)n_positions, a.q_gain = q_gain, a.k_gain = k_gain;
  a.eps = d->eps, a.q_out = q_out, a.status = status_word;
  return a;
}

}  // namespace

phyai_status_t check_paged(const phyai_paged_cache_t* c, uint32_t layer, uint32_t batch, const int32_t* cu, const int32_t* kv_lens,
                           const int32_t* table, uint32_t max_pages, uint32_t tokens, bool all_layers, PagedBatch* out) {
  if (!c || c->struct_size != sizeof(phyai_paged_cache_t)) return bad_arg("cache is NULL or has a wrong struct_size");
  if (!c->pages || !c->n_layers || !c->n_kv_heads || !c->n_pages) return bad_arg("pages is NULL or a size of the cache is zero");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) {
    snprintf(g_paged_err, sizeof(g_paged_err), "head_dim must be 64, 128 or 256");
    return PHYAI_ERR_UNSUPPORTED;
  }
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) {
    snprintf(g_paged_err, sizeof(g_paged_err), "page_size must be 16, 32, 64, 128 or 256");
    return PHYAI_ERR_UNSUPPORTED;
  }
  if (c->dtype != PHYAI_F32 && c->dtype != PHYAI_BF16) {
    snprintf(g_paged_err, sizeof(g_paged_err), "the cache's type must be float32 or bfloat16");
    return PHYAI_ERR_UNSUPPORTED;
  }
  if (!aligned16(c->pages)) return bad_arg("pages must be 16-byte aligned");
  if (c->n_kv_heads > 65535u || c->n_layers > 32767u || c->n_pages * c->page_size > 0x7fffffffull) return bad_arg("the cache is too large");
  if (!all_layers && layer >= c->n_layers) return bad_arg("layer out of range");
  if (!batch || batch > (uint32_t)PAGED_MAX_BATCH) return bad_arg("batch must be 1..1024");
  if ((!all_layers && !cu) || !kv_lens || !table || !max_pages) return bad_arg("cu_q_lens, kv_lens or page_table is NULL, or max_pages is 0");
  if (!aligned4(cu) || !aligned4(kv_lens) || !aligned4(table)) return bad_arg("cu_q_lens, kv_lens and page_table must be 4-byte aligned");
  if (tokens > 0x7fffffffu || (uint64_t)max_pages * c->page_size > PAGED_MAX_KEYS) return bad_arg("tokens or max_pages too large");
  out->cu = cu, out->kv_lens = kv_lens, out->table = table, out->batch = (int)batch, out->tokens = (int)tokens, out->max_pages = (int)max_pages;
  out->page_shift = __builtin_ctz(c->page_size), out->n_pages = (int)c->n_pages;
  return PHYAI_OK;
}

}  // namespace phyai

extern "C" {

const char* phyai_paged_last_error(void) { return phyai::g_paged_err; }

phyai_status_t phyai_norm_rope_heads(const phyai_heads_desc_t* desc, uint32_t tokens, const void* q, uint64_t q_stride, const void* k,
                                     uint64_t k_stride, const int32_t* positions, const float* rope_cos_sin, uint64_t n_positions,
                                     const float* q_gain, const float* k_gain, void* q_out, void* k_out, int32_t* status_word, void* stream) {
  using namespace phyai;
  phyai_status_t s = check_heads(desc, tokens, q, q_stride, k, k_stride, rope_cos_sin, n_positions, q_gain, k_gain, q_out, status_word);
  if (s != PHYAI_OK) return s;
  if (tokens && (!k_out || (rope_cos_sin && !positions))) return bad_arg("k_out is NULL, or positions is NULL with a rotation");
  if (!aligned16(k_out) || !aligned4(positions)) return bad_arg("pointers and row strides must be multiples of 16 bytes, positions of 4");
  if (!tokens) return PHYAI_OK;
  HeadsArgs a = heads_args(desc, tokens, q, q_stride, k, k_stride, positions, rope_cos_sin, n_positions, q_gain, k_gain, q_out, status_word);
  a.k_out = k_out;
  if (const cudaError_t e = paged_call(status_word, &a.pb); e != cudaSuccess) return launch_result(e);
  return launch_result(dispatch_heads<false>((int)desc->head_dim, desc->in_dtype, desc->out_dtype, a, reinterpret_cast<cudaStream_t>(stream)));
}

phyai_status_t phyai_append_paged_kv(const phyai_paged_cache_t* cache, const phyai_heads_desc_t* desc, uint32_t layer, uint32_t tokens,
                                     const void* q, uint64_t q_stride, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride,
                                     uint32_t batch, const int32_t* cu_q_lens, const int32_t* kv_lens, const int32_t* page_table,
                                     uint32_t max_pages, const int32_t* positions, const float* rope_cos_sin, uint64_t n_positions,
                                     const float* q_gain, const float* k_gain, void* q_out, int32_t* status_word, void* stream) {
  using namespace phyai;
  phyai_status_t s = check_heads(desc, tokens, q, q_stride, k, k_stride, rope_cos_sin, n_positions, q_gain, k_gain, q_out, status_word);
  if (s != PHYAI_OK) return s;
  HeadsArgs a = heads_args(desc, tokens, q, q_stride, k, k_stride, positions, rope_cos_sin, n_positions, q_gain, k_gain, q_out, status_word);
  s = check_paged(cache, layer, batch, cu_q_lens, kv_lens, page_table, max_pages, tokens, false, &a.pb);
  if (s != PHYAI_OK) return s;
  if (cache->n_kv_heads != desc->n_kv_heads || cache->head_dim != desc->head_dim || cache->dtype != desc->out_dtype)
    return bad_arg("heads, head_dim or type of desc differ from the cache's");
  const uint64_t es = desc->in_dtype == PHYAI_F32 ? 4 : 2;
  if (tokens && !v) return bad_arg("a pointer argument is NULL");
  if (v_stride < (uint64_t)desc->n_kv_heads * desc->head_dim || v_stride > (1ull << 40)) return bad_arg("a row stride is smaller than the row's heads, or too large");
  if (!aligned16(v) || (v_stride * es) % 16 || !aligned4(positions)) return bad_arg("pointers and row strides must be multiples of 16 bytes, positions of 4");
  if (!tokens) return PHYAI_OK;
  a.v = v, a.v_stride = (long long)v_stride;
  if (const cudaError_t e = paged_call(status_word, &a.pb); e != cudaSuccess) return launch_result(e);
  const size_t plane = (size_t)cache->n_pages * cache->page_size * cache->n_kv_heads * cache->head_dim * (cache->dtype == PHYAI_F32 ? 4 : 2);
  a.k_plane = (char*)cache->pages + 2 * (size_t)layer * plane, a.v_plane = (char*)a.k_plane + plane;
  return launch_result(dispatch_heads<true>((int)desc->head_dim, desc->in_dtype, desc->out_dtype, a, reinterpret_cast<cudaStream_t>(stream)));
}

phyai_status_t phyai_pack_paged_kv(const phyai_paged_cache_t* cache, uint32_t batch, const int32_t* kv_lens, const int32_t* page_table,
                                   uint32_t max_pages, void* prefix_kv, uint64_t kv_tokens, int32_t* cu_prefix_lens, int32_t* status_word,
                                   void* stream) {
  using namespace phyai;
  PagedBatch p{};
  phyai_status_t s = check_paged(cache, 0, batch, nullptr, kv_lens, page_table, max_pages, 0, true, &p);
  if (s != PHYAI_OK) return s;
  if ((!prefix_kv && kv_tokens) || !cu_prefix_lens || !status_word) return bad_arg("a pointer argument is NULL");
  if (!aligned16(prefix_kv) || !aligned4(cu_prefix_lens) || !aligned4(status_word)) return bad_arg("prefix_kv must be 16-byte aligned, cu_prefix_lens and status_word 4-byte");
  const size_t row_bytes = (size_t)cache->n_kv_heads * cache->head_dim * (cache->dtype == PHYAI_F32 ? 4 : 2), chunks = row_bytes / 16;
  const size_t longest = (size_t)max_pages * cache->page_size < kv_tokens ? (size_t)max_pages * cache->page_size : kv_tokens;
  if (kv_tokens > 0x7fffffffull || (size_t)max_pages * cache->page_size * chunks > 0x7fffffffull) return bad_arg("kv_tokens or max_pages too large");
  const uint64_t o = reinterpret_cast<uintptr_t>(prefix_kv), o_bytes = 2ull * cache->n_layers * kv_tokens * row_bytes;
  const uint64_t i = reinterpret_cast<uintptr_t>(cache->pages), i_bytes = 2ull * cache->n_layers * cache->n_pages * cache->page_size * row_bytes;
  if (o < i + i_bytes && i < o + o_bytes) return bad_arg("prefix_kv overlaps the pages");
  if (const cudaError_t e = paged_call(status_word, &p); e != cudaSuccess) return launch_result(e);
  // (a block per chunk of a request of twice the average length; the blocks of longer ones take several: a table is as wide as the longest
  // request may become, and blocks without work are not free)
  const size_t likely = 2 * kv_tokens / batch + 64, gx = ((longest < likely ? longest : likely) * chunks + PP_CHUNK - 1) / PP_CHUNK;
  return launch_result(launch_pdl(k_pack_pages, dim3((unsigned)(gx ? gx : 1), cache->n_layers * 2, batch), dim3(PP_T), 0, reinterpret_cast<cudaStream_t>(stream),
                                  (const uint4*)cache->pages, (uint4*)prefix_kv, cu_prefix_lens, status_word, p, (long long)kv_tokens, (int)chunks));
}

}  // extern "C"
