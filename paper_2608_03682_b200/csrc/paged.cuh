// Paged cache of keys and values: what its operators share (paged_heads.cu writes and drains it, paged_attention*.cu read it).
//
// The pool is [n_layers][2 (K, V)][n_pages * page_size][n_kv_heads][head_dim], head_dim contiguous: the layout of the denoising
// loop's prefix cache, so that one page number serves all layers and both planes.  Cached token t of request b is row
// table[b][t / page_size] * page_size + t % page_size of every plane.  Requests are ragged: request b's new tokens are rows
// cu[b] .. cu[b + 1] - 1 of a call's token rows, its cache holds kv_lens[b] tokens of which the new ones are the last.
#pragma once

#include "../../include/phyai.h"
#include "kernels.h"
#include "ptx.cuh"

namespace phyai {

constexpr int PAGED_MAX_BATCH = 1024;
constexpr uint64_t PAGED_MAX_KEYS = 0x7fffff00ull;      // of a request: the kernels round a length up to tiles of keys, in 32 bits

struct PagedBatch {
  const int* cu;          // [batch + 1]
  const int* kv_lens;     // [batch]
  const int* table;       // [batch][max_pages]
  int batch, tokens, max_pages;
  int page_shift;         // log2(page_size)
  int n_pages;
  unsigned* raised_by;    // which call raised this call's status word for an entry, and this call (see paged_stopped)
  unsigned call;
};

// The status word.  A call that finds it up writes nothing, but an entry that names no page (or a position outside the rotary table)
// concerns one request alone: the others' blocks, which may begin after the word went up, and the merge go on.  So whoever raises the word for an
// entry notes the call's number first, and blocks that find the word up look whether it was their own call.  The word itself stays what a
// caller expects, and while it is down nothing more is read.  (Notes lie in a table of the device by the word's address, paged_call: two calls on
// words that share a note, and that both meet such entries at a time, could at worst take their own word for an earlier call's.)
__device__ __forceinline__ bool paged_stopped(const int* status, const PagedBatch& p) {
  const int v = *reinterpret_cast<const volatile int*>(status);
  if (v == ST_OK) return false;
  if (v != ST_INVALID_ARG) return true;
  __threadfence();
  return *reinterpret_cast<const volatile unsigned*>(p.raised_by) != p.call;
}
__device__ __forceinline__ void paged_bad_entry(int* status, const PagedBatch& p) {
  atomicExch(p.raised_by, p.call);
  __threadfence();
  atomicCAS(status, ST_OK, ST_INVALID_ARG);
}
// for lengths out of order (every block sees them by itself) and in calls that do not read the word: stops every other call
__device__ __forceinline__ void paged_raise(int* status, const PagedBatch& p) {
  atomicExch(p.raised_by, 0u);
  __threadfence();
  atomicExch(status, ST_INVALID_ARG);
}

// row of the planes that holds cached token t of request b, or -1 if its table entry names no page
__device__ __forceinline__ long long paged_row(const PagedBatch& p, int b, int t) {
  const int page = p.table[(size_t)b * p.max_pages + (t >> p.page_shift)];
  if ((unsigned)page >= (unsigned)p.n_pages) return -1;
  return ((long long)page << p.page_shift) + (t & ((1 << p.page_shift) - 1));
}

// Whether entry i of the lengths is in order (i = 0 .. batch - 1): the token rows do not go backwards or past the call's, the
// cached tokens fit the table, and (append) the new ones are among them.
__device__ __forceinline__ bool paged_entry_bad(const PagedBatch& p, int i, int lo, int hi, int kv, bool new_in_cache) {
  return lo < 0 || hi < lo || hi > p.tokens || kv < 0 || (long long)kv > ((long long)p.max_pages << p.page_shift) || (new_in_cache && hi - lo > kv);
}

// Attention over the pages: row r of a request's packed rows is its new token r / group at query head kv_head * group + r % group
// (the query heads that share a kv head stand together, so that they share the keys that a tile fetches).
struct PagedAttn {
  PagedBatch pb;
  const void* q;          // [tokens] rows of hq heads, q_stride elements apart
  long long q_stride;
  void* out;              // [tokens][hq][dh]
  const void *k_plane, *v_plane;
  int plane;              // of K, among all planes of the pool (V: the next one)
  const int* prefix_lens; // [batch] or null
  int causal, hq, hkv, group;
  float scale_log2;       // softmax scale * log2(e)
  int ranges;             // most key ranges of a row
  float* part_o;          // [ranges][tokens][hq][dh]: unnormalised accumulators of a key range
  float4* part_ml;        // [ranges][tokens][hq]: maximum (log2 units), sum, ranges of this row, 1 if it sees a key
  int* status;
  unsigned wait_limit;
};

// 1 / (sum of a row's weights); 0 for a row that sees no key.  (A row all of whose keys have the logit -infinity sums to 0: its result is 0 / 0, NaN.)
__device__ __forceinline__ float paged_inv(float sum, bool sees) { return sees ? 1.0f / sum : 0.f; }

// A request's lengths, and how many keys its new token i sees: keys [0, limit).
struct PagedRequest {
  int b, lo, n, kv, prefix;
  __device__ __forceinline__ int limit(int i, int causal) const { return causal ? min(kv, max(max(kv - n + i + 1, prefix), 0)) : kv; }
};

// Request and row tile of unit `unit` (tiles of RT packed rows, requests in order); also whether every length of the call is in
// order.  By a whole warp; r.b = -1: there are fewer units.
template <int RT>
__device__ __forceinline__ bool paged_unit(const PagedAttn& a, int unit, PagedRequest& r, int& tile) {
  const int lane = threadIdx.x & 31;
  bool bad = false;
  int acc = 0;
  r.b = -1, r.lo = r.n = r.kv = r.prefix = 0, tile = 0;
  for (int i0 = 0; i0 < a.pb.batch; i0 += 128) {      // (128 requests' lengths on their way at a time)
    int lo[4], hi[4], kv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + 32 * j + lane;
      lo[j] = hi[j] = kv[j] = 0;
      if (i < a.pb.batch) lo[j] = a.pb.cu[i], hi[j] = a.pb.cu[i + 1], kv[j] = a.pb.kv_lens[i];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + 32 * j >= a.pb.batch) break;
      const bool wrong = i0 + 32 * j + lane < a.pb.batch && paged_entry_bad(a.pb, i0 + 32 * j + lane, lo[j], hi[j], kv[j], false);
      bad |= wrong;
      const int n = wrong ? 0 : ((hi[j] - lo[j]) * a.group + RT - 1) / RT;
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, acc + incl > unit);
      if (r.b < 0 && hit) {
        const int src = __ffs(hit) - 1;
        r.b = i0 + 32 * j + src, r.lo = __shfl_sync(0xffffffffu, lo[j], src), r.n = __shfl_sync(0xffffffffu, hi[j], src) - r.lo;
        r.kv = __shfl_sync(0xffffffffu, kv[j], src);
        tile = unit - acc - __shfl_sync(0xffffffffu, incl - n, src);
      }
      acc += __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  if (__any_sync(0xffffffffu, bad)) return false;
  if (r.b >= 0 && a.prefix_lens) r.prefix = min(max(a.prefix_lens[r.b], 0), r.kv);
  return true;
}

// Whether a value of keys [k0, k1) that a row does not see is infinite or NaN, in channels [c0, c0 + 32 C).  By a whole warp, C channels a lane.
template <int C, typename T>
__device__ __noinline__ bool paged_hidden_odd(const PagedAttn& a, int b, int hk, int dh, int c0, int k0, int k1) {
  bool odd = false;
  for (int k = k0; k < k1; ++k) {
    const long long row = paged_row(a.pb, b, k);
    if (row < 0) continue;
    const T* v = (const T*)a.v_plane + ((size_t)row * a.hkv + hk) * dh + c0 + (threadIdx.x & 31) * C;
#pragma unroll
    for (int i = 0; i < C; ++i) odd |= !(fabsf(to_float(v[i])) < INFINITY);
  }
  return __any_sync(0xffffffffu, odd);
}

// One row over keys [k0, k1) of its request, key by key: the result of rows whose tile's products met an infinity or a NaN of a key
// that the row does not see (0 x infinity).  By a whole warp; lane: channels lane * DH / 32 on.  o is unnormalised.
template <int DH, typename T>
__device__ __noinline__ void paged_row_alone(const PagedAttn& a, int b, const T* q, int hk, int k0, int k1, float* o, float& m, float& l) {
  constexpr int C = DH / 32;
  const int c = (threadIdx.x & 31) * C;
  float x[C];
#pragma unroll
  for (int i = 0; i < C; ++i) x[i] = to_float(q[c + i]), o[i] = 0.f;
  m = -INFINITY, l = 0.f;
#pragma unroll 4
  for (int k = k0; k < k1; ++k) {
    const long long row = paged_row(a.pb, b, k);
    if (row < 0) continue;
    const size_t at = ((size_t)row * a.hkv + hk) * DH + c;
    const T *kp = (const T*)a.k_plane + at, *vp = (const T*)a.v_plane + at;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) s = fmaf(x[i], to_float(kp[i]), s);
    s = warp_sum(s) * a.scale_log2;
    const float mn = fmaxf(m, s), sub = mn == -INFINITY ? 0.f : mn, corr = exp2f(m - sub), p = exp2f(s - sub);
    l = fmaf(l, corr, p), m = mn;
#pragma unroll
    for (int i = 0; i < C; ++i) o[i] = fmaf(p, to_float(vp[i]), o[i] * corr);
  }
}

// The checks that every operator on a paged cache makes of it and of a call's requests (message in g_paged_err).
extern thread_local char g_paged_err[256];
phyai_status_t check_paged(const phyai_paged_cache_t* c, uint32_t layer, uint32_t batch, const int32_t* cu, const int32_t* kv_lens,
                           const int32_t* table, uint32_t max_pages, uint32_t tokens, bool all_layers, PagedBatch* out);
int paged_sm_count();
// numbers the call and finds the note of its status word on the current device
cudaError_t paged_call(const int32_t* status_word, PagedBatch* p);

// Key ranges of a row tile: at least `least` tiles of keys each.
__host__ __device__ __forceinline__ int ranges_of(int tiles, int most, int least) {
  const int r = tiles / least < most ? tiles / least : most;
  return r > 1 ? r : 1;
}
// the pool as rows of 64 channels: {64, rows of a plane, blocks of 64 channels in a row, planes}; a copy: `rows` rows, `blocks` blocks
bool paged_pool_map(void* map, const phyai_paged_cache_t* c, uint32_t rows, uint32_t blocks);

// many rows: paged_attention_pair.cu
constexpr int PAGED_PAIR_MERGE = 7;                     // time that splitting units costs (fp32 results, a second kernel), in tiles of 128 keys
bool paged_pair_supported(int dh, int group);
int paged_pair_tokens(int group);                       // tokens of a unit
int paged_pair_resident(int dh);                        // pairs at a time (0 on an error)
cudaError_t launch_paged_pair(const PagedAttn& a, const phyai_paged_cache_t* cache, long long items, cudaStream_t st);

}  // namespace phyai
