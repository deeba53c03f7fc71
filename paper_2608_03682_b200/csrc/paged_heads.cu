// What writes and drains the paged cache, and the heads' norm and rotation on their own:
//   phyai_norm_rope_heads   q, k rows -> normed, rotated rows
//   phyai_append_paged_kv   the same for k, written into the pages with v; q rows in the same pass when given
//   phyai_pack_paged_kv     pages -> the ragged prefix cache that the denoising loop reads
//
// A head x of dh channels becomes  y = x * rsqrt(mean(x^2) + eps) * (1 + gain)  and then, for j < dh / 2,
//   (y_j, y_{j + dh/2}) -> (y_j cos - y_{j + dh/2} sin, y_{j + dh/2} cos + y_j sin)  with the table's row of its position.
// Everything is read once and written once, so memory bounds it: a group of dh / 8 lanes takes a head, 8 channels a lane (16-byte
// accesses of bf16), the sum of squares and the rotary partner come by shuffles (the partner channels sit dh / 16 lanes away), and the
// arithmetic is fp32 with one rounding at the store.
#include <cstdio>

#include "../../include/phyai.h"
#include "paged.cuh"

namespace phyai {

thread_local char g_paged_err[256] = "";

namespace {

// 8 consecutive channels
struct F8 {
  float v[8];
};
__device__ __forceinline__ F8 load8(const float* p) {
  F8 r;
  *reinterpret_cast<float4*>(r.v) = *reinterpret_cast<const float4*>(p);
  *reinterpret_cast<float4*>(r.v + 4) = *reinterpret_cast<const float4*>(p + 4);
  return r;
}
__device__ __forceinline__ F8 load8(const __nv_bfloat16* p) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  F8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[2 * i] = __uint_as_float(u[i] << 16), r.v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  return r;
}
__device__ __forceinline__ void store8(float* p, const F8& x) {
  *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(x.v);
  *reinterpret_cast<float4*>(p + 4) = *reinterpret_cast<const float4*>(x.v + 4);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const F8& x) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x.v[2 * i], x.v[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
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

constexpr int HT = 256;                  // threads of a block

// A warp takes a token's heads, 32 / (dh / 8) at a time (a "slot" is such a set); a unit is U slots of one token, whose loads are all
// issued before the first is used.
template <int DH, typename IN, typename OUT, bool APPEND, int U>
__global__ void __launch_bounds__(HT) k_heads(const HeadsArgs a) {
  constexpr int LANES = DH / 8, HPS = 32 / LANES;           // lanes per head, heads per slot
  __shared__ int s_cu[APPEND ? PAGED_MAX_BATCH + 1 : 1], s_kv[APPEND ? PAGED_MAX_BATCH : 1];
  __shared__ int s_skip;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LANES, c = (lane % LANES) * 8;
  const int H = (a.q ? a.hq : 0) + a.hkv + (a.v ? a.hkv : 0), hq = a.q ? a.hq : 0;
  const int slots = (H + HPS - 1) / HPS, units_t = (slots + U - 1) / U;      // per token
  const long long units = (long long)a.tokens * units_t;
  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x == 0) s_skip = status_set(a.status);
  if constexpr (APPEND) {
    bool bad = false;
    for (int i = threadIdx.x; i < a.pb.batch; i += HT) {
      const int lo = a.pb.cu[i], hi = a.pb.cu[i + 1], kv = a.pb.kv_lens[i];
      bad |= paged_entry_bad(a.pb, i, lo, hi, kv, true);
      s_cu[i] = lo, s_kv[i] = kv;
      if (i + 1 == a.pb.batch) s_cu[i + 1] = hi;
    }
    bad = __syncthreads_or(bad);
    if (bad) {
      if (threadIdx.x == 0) atomicExch(a.status, ST_INVALID_ARG);
      return;
    }
  } else {
    __syncthreads();
  }
  if (s_skip) return;
  const IN* const src[3] = {(const IN*)a.q, (const IN*)a.k, (const IN*)a.v};

  for (long long unit = (long long)blockIdx.x * (HT / 32) + warp; unit < units; unit += (long long)gridDim.x * (HT / 32)) {
    const int tok = (int)(unit / units_t), slot0 = (int)(unit - (long long)tok * units_t) * U;
    F8 x[U];
    int head[U], kind[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = (slot0 + u) * HPS + sub;
      kind[u] = h < hq ? 0 : h < hq + a.hkv ? 1 : h < H ? 2 : 3;
      head[u] = kind[u] == 0 ? h : kind[u] == 1 ? h - hq : h - hq - a.hkv;
      if (kind[u] < 3) {
        const long long stride = kind[u] == 0 ? a.q_stride : kind[u] == 1 ? a.k_stride : a.v_stride;
        x[u] = load8((kind[u] == 0 ? src[0] : kind[u] == 1 ? src[1] : src[2]) + tok * stride + head[u] * DH + c);
      } else {
        x[u] = F8{};
      }
    }
    // ---- where the token is
    int pos = 0;
    long long row = -1;
    bool ok = true;
    if constexpr (APPEND) {
      int before = 0;                                        // requests that end at or before this token
      for (int i0 = 0; i0 < a.pb.batch; i0 += 32) before += __popc(__ballot_sync(0xffffffffu, i0 + lane < a.pb.batch && s_cu[i0 + lane + 1] <= tok));
      const int b = before;
      if (tok < s_cu[0] || b >= a.pb.batch) continue;        // (a row of no request)
      const int place = s_kv[b] - (s_cu[b + 1] - tok);
      row = paged_row(a.pb, b, place);
      pos = a.positions ? a.positions[tok] : place;
      ok = row >= 0;
    } else {
      if (a.positions) pos = a.positions[tok];
    }
    if (a.rope && (unsigned)pos >= (unsigned)a.n_positions) ok = false;
    if (!ok) {                                               // (the whole warp: nothing of this token is written)
      if (lane == 0) atomicExch(a.status, ST_INVALID_ARG);
      continue;
    }
    float cs[8], sn[8];
    if (a.rope) {
      const float4* t = reinterpret_cast<const float4*>(a.rope + ((size_t)pos * (DH / 2) + (c & (DH / 2 - 1))) * 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 w = __ldg(t + i);
        cs[2 * i] = w.x, sn[2 * i] = w.y, cs[2 * i + 1] = w.z, sn[2 * i + 1] = w.w;
      }
      if (c < DH / 2) {                                      // y_j cos - y_{j + dh/2} sin in the lower half
#pragma unroll
        for (int i = 0; i < 8; ++i) sn[i] = -sn[i];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* gain = kind[u] == 0 ? a.q_gain : kind[u] == 1 ? a.k_gain : nullptr;
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[u].v[i], x[u].v[i], ss);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (gain) {
        const float r = rsqrtf(ss * (1.0f / DH) + a.eps);
        const F8 g = load8(gain + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u].v[i] *= r * (1.0f + g.v[i]);
      }
      if (a.rope) {
        F8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y.v[i] = __shfl_xor_sync(0xffffffffu, x[u].v[i], LANES / 2);
        if (kind[u] < 2) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u].v[i] = fmaf(y.v[i], sn[i], x[u].v[i] * cs[i]);
        }
      }
      if (kind[u] == 0) {
        store8((OUT*)a.q_out + ((size_t)tok * a.hq + head[u]) * DH + c, x[u]);
      } else if (kind[u] < 3) {
        OUT* base = APPEND ? (OUT*)(kind[u] == 1 ? a.k_plane : a.v_plane) : (OUT*)a.k_out;
        store8(base + ((size_t)(APPEND ? row : tok) * a.hkv + head[u]) * DH + c, x[u]);
      }
    }
  }
}

}  // namespace

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
  constexpr int HPS = 32 / (DH / 8), U = 4;
  const int H = (a.q ? a.hq : 0) + a.hkv + (a.v ? a.hkv : 0), slots = (H + HPS - 1) / HPS, n_sm = paged_sm_count();
  if (n_sm <= 0) return cudaErrorInvalidDevice;
  const long long per_warp = (long long)a.tokens * slots;
  // Few tokens: a warp per slot, all of them at a time; many: four slots a warp.
  if (per_warp <= (long long)n_sm * 16)
    return launch_pdl(k_heads<DH, IN, OUT, APPEND, 1>, dim3((unsigned)((per_warp + HT / 32 - 1) / (HT / 32))), dim3(HT), 0, st, a);
  const long long units = (long long)a.tokens * ((slots + U - 1) / U), blocks = (units + HT / 32 - 1) / (HT / 32);
  const long long most = (long long)n_sm * 8;
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

// Pages -> packed rows.  Blocks move 16 KB of one plane (grid.y) and request (grid.z), four 16-byte loads a thread; every block adds up
// the lengths before its request itself.
constexpr int PP_T = 256, PP_U = 4, PP_CHUNK = PP_T * PP_U;
__global__ void __launch_bounds__(PP_T) k_pack_pages(const uint4* pages, uint4* dst, int* cu, int* status, const PagedBatch p, long long kv_tokens,
                                                     int row_chunks) {
  __shared__ long long s_part[2][PP_T / 32];
  __shared__ int s_skip;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.z;
  pdl_launch_dependents();
  pdl_wait();
  if (tid == 0) s_skip = status_set(status);
  const int my_len = p.kv_lens[b];
  const bool first = blockIdx.x == 0 && blockIdx.y == 0;
  const int page_chunks = row_chunks << p.page_shift;
  const int i0 = (int)blockIdx.x * PP_CHUNK + tid;
  const bool in_range = my_len >= 0 && (long long)my_len <= ((long long)p.max_pages << p.page_shift);
  const int n = in_range ? my_len * row_chunks : 0;
  if ((int)blockIdx.x * PP_CHUNK >= n && !first) return;
  const size_t plane_chunks = ((size_t)p.n_pages << p.page_shift) * row_chunks;
  const uint4* src = pages + (size_t)blockIdx.y * plane_chunks;
  uint4 x[PP_U];
  bool have[PP_U], bad_page = false;
#pragma unroll
  for (int u = 0; u < PP_U; ++u) {
    const int i = i0 + u * PP_T;
    have[u] = false;
    if (i < n) {
      const int pg = i / page_chunks, page = p.table[(size_t)b * p.max_pages + pg];
      have[u] = (unsigned)page < (unsigned)p.n_pages;
      bad_page |= !have[u];
      if (have[u]) x[u] = __ldcs(src + (size_t)page * page_chunks + (i - pg * page_chunks));
    }
  }
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
  if (first && tid == 0) {
    if (b == 0) cu[0] = 0;
    cu[b + 1] = (int)min(before + max(my_len, 0), 0x7fffffffLL);
    if (bad) atomicExch(status, ST_INVALID_ARG);
  }
  if (bad) return;
  if (bad_page) atomicExch(status, ST_INVALID_ARG);
  uint4* o = dst + ((size_t)blockIdx.y * kv_tokens + before) * row_chunks + i0;
#pragma unroll
  for (int u = 0; u < PP_U; ++u)
    if (have[u]) o[u * PP_T] = x[u];
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
  if (tokens > 0x7fffffffu || (uint64_t)max_pages * c->page_size > 0x7fffffffull) return bad_arg("tokens or max_pages too large");
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
  if (!aligned16(k_out)) return bad_arg("pointers and row strides must be multiples of 16 bytes");
  if (!tokens) return PHYAI_OK;
  HeadsArgs a = heads_args(desc, tokens, q, q_stride, k, k_stride, positions, rope_cos_sin, n_positions, q_gain, k_gain, q_out, status_word);
  a.k_out = k_out;
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
  if (!aligned16(v) || (v_stride * es) % 16) return bad_arg("pointers and row strides must be multiples of 16 bytes");
  if (!tokens) return PHYAI_OK;
  a.v = v, a.v_stride = (long long)v_stride;
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
  if (!aligned16(prefix_kv)) return bad_arg("prefix_kv must be 16-byte aligned");
  const size_t row_bytes = (size_t)cache->n_kv_heads * cache->head_dim * (cache->dtype == PHYAI_F32 ? 4 : 2), chunks = row_bytes / 16;
  const size_t longest = (size_t)max_pages * cache->page_size < kv_tokens ? (size_t)max_pages * cache->page_size : kv_tokens;
  if (kv_tokens > 0x7fffffffull || (size_t)max_pages * cache->page_size * chunks > 0x7fffffffull) return bad_arg("kv_tokens or max_pages too large");
  const size_t gx = (longest * chunks + PP_CHUNK - 1) / PP_CHUNK;
  return launch_result(launch_pdl(k_pack_pages, dim3((unsigned)(gx ? gx : 1), cache->n_layers * 2, batch), dim3(PP_T), 0, reinterpret_cast<cudaStream_t>(stream),
                                  (const uint4*)cache->pages, (uint4*)prefix_kv, cu_prefix_lens, status_word, p, (long long)kv_tokens, (int)chunks));
}

}  // extern "C"
