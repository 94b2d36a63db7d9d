// The paged cache in 8 bits: quantising new tokens into it, gathering kept tokens into fewer pages, copying pages.
#include <float.h>

#include "cache.h"

namespace spindle {

spindle_status check_cache(const spindle_cache *c, CacheView *out) {
  if (!c) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_pages < 1 || c->n_kv_heads < 1) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "n_pages and n_kv_heads must be >= 1");
  if (c->head_dim != kHeadDim) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "head_dim must be 128, got %d", c->head_dim);
  if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256)
    SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "page_tokens must be 32, 64, 128 or 256, got %d", c->page_tokens);
  if (c->format != SPINDLE_E4M3 && c->format != SPINDLE_I8) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "unknown cache format %d", c->format);
  if ((int64_t)c->n_pages * c->n_kv_heads >= (1 << 30)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "n_pages * n_kv_heads must be below 2^30");
  if (c->n_kv_heads > 1024) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "n_kv_heads must be <= 1024");
  if (!c->k || !c->v || !c->k_scale || !c->v_scale)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "the cache's k, v, k_scale and v_scale are required");
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "the cache's k and v must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale) | reinterpret_cast<uintptr_t>(c->pos)) & 3)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "the cache's scales and positions must be 4-byte aligned");
  *out = CacheView{static_cast<uint8_t *>(c->k), static_cast<uint8_t *>(c->v), c->k_scale, c->v_scale, c->pos,
                   c->n_pages, c->n_kv_heads, c->page_tokens, __builtin_ctz((unsigned)c->page_tokens)};
  return SPINDLE_OK;
}

spindle_status check_table(const void *table, int32_t width, const void *len, int32_t batch, const CacheView &c) {
  if (!table || !len) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "table and len are required");
  if (batch < 1 || width < 1) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "batch and the table's width must be >= 1");
  if (batch > 32767) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "batch must be <= 32767");
  if ((int64_t)width * c.P > (1 << 30)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "a table's row may hold at most 2^30 tokens");
  return SPINDLE_OK;
}

namespace {

constexpr int kPer = 8;                         // dimensions per thread
constexpr int kQuad = 4;                        // tokens per thread
constexpr int kAcross = kHeadDim / kPer;        // threads side by side on a row

// Largest value over the block; every thread gets it.
__device__ __forceinline__ float block_max(float v, float *shared) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  if (lane_id() == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  const int waves = blockDim.x >> 6;
  v = shared[0];
  for (int w = 1; w < waves; ++w) v = fmaxf(v, shared[w]);
  return v;
}

template <int DT>
__device__ __forceinline__ void load8(const char *p, float *x) {
  typedef typename Elem<DT>::type T;
  u4 raw[sizeof(T) / 2];
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const u4 *>(p)[i];
  const T *e = reinterpret_cast<const T *>(raw);
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = Elem<DT>::to_float(e[i]);
}

struct AppendArgs {
  CacheView c;
  const int32_t *table, *len, *cu, *positions;
  const char *K, *V;
  long long sb, sh, st;                         // bytes
  int width, max_new, rows, total_new, tiles;   // rows: of K and V behind one pointer
};

// One workgroup of 4 P threads writes one page of one head of K or V: a thread holds 8 dimensions of 4 tokens, so the page
// stays in registers between its largest magnitude and its codes, and the input is read once.  Bound by memory where it
// is a prompt (32768 f16 tokens of 8 heads, 201 MB: 39 us, 5.1 TB/s with part of it cached, 47 with nothing cached; a large
// copy reaches 4.8), by four trips to memory that wait for each other where it is a step (64 sequences, one token: 6.3 us).
template <int DT, int FMT>
__global__ void cache_append(AppendArgs a) {
  __shared__ float part[16];
  const CacheView &c = a.c;
  int id = blockIdx.x;
  const bool is_v = id & 1;
  id >>= 1;
  const int head = id % c.H;
  id /= c.H;
  const int tile = id % a.tiles, b = id / a.tiles;
  const int n = min(max(a.len[b], 0), a.width * c.P);
  int row0 = 0, m = a.max_new;
  if (a.cu) {
    row0 = a.cu[b];
    m = min(max(a.cu[b + 1] - row0, 0), a.max_new);
  }
  const int begin = (n / c.P + tile) * c.P;                         // first token of the page
  const int lo = max(n, begin);
  const int hi = (int)min(min((long long)n + m, (long long)begin + c.P), (long long)a.width * c.P);
  if (lo >= hi) return;
  const int page = a.table[(size_t)b * a.width + begin / c.P];
  if (page < 0 || page >= c.n_pages) return;
  const char *src = (is_v ? a.V : a.K) + (a.cu ? 0 : (size_t)b * a.sb) + (size_t)head * a.sh;
  uint8_t *codes = (is_v ? c.v : c.k) + page_row(c, page, head) * kHeadDim;
  float *scale_at = (is_v ? c.vs : c.ks) + (size_t)page * c.H + head;
  const int across = threadIdx.x % kAcross, slot0 = threadIdx.x / kAcross * kQuad;
  float x[kQuad][kPer];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < kQuad; ++i) {
    const int g = begin + slot0 + i;
    const long long row = (long long)row0 + (g - n);
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[i][j] = 0.f;
    if (g >= lo && g < hi && row >= 0 && row < a.rows)
      load8<DT>(src + row * a.st + (size_t)across * kPer * sizeof(typename Elem<DT>::type), x[i]);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const float m1 = __builtin_fabsf(x[i][j]);
      amax = fmaxf(amax, m1 < INFINITY ? m1 : 0.f);                  // NaN and infinities do not set the scale
    }
  }
  const float had = lo > begin ? *scale_at : 0.f;
  amax = block_max(amax, part);
  const float s = fmaxf(had, Code<FMT>::scale_for(amax));
  const bool whole = s != had;                                       // a page that begins, or whose scale grows, is written whole
  const float rs = 1.f / s;
#pragma unroll
  for (int i = 0; i < kQuad; ++i) {
    const int g = begin + slot0 + i;
    u2 *at = reinterpret_cast<u2 *>(codes + (size_t)(slot0 + i) * kHeadDim + across * kPer);
    if (g >= lo && g < hi) {
      *at = u2{Code<FMT>::encode4(x[i], s, rs), Code<FMT>::encode4(x[i] + 4, s, rs)};
    } else if (whole) {
      u2 w = {0, 0};
      if (g < lo) {
        w = *at;
        w = u2{Code<FMT>::rescale4(w[0], had, s), Code<FMT>::rescale4(w[1], had, s)};
      }
      *at = w;
    }
  }
  if (threadIdx.x == 0 && whole) *scale_at = s;
  if (c.pos && !is_v && across == 0) {
#pragma unroll
    for (int i = 0; i < kQuad; ++i) {
      const int g = begin + slot0 + i;
      if (g < lo || g >= hi) continue;
      const long long row = (a.cu ? (long long)row0 : (long long)b * a.max_new) + (g - n);
      c.pos[page_row(c, page, head) + slot0 + i] = a.positions && row >= 0 && row < a.total_new ? a.positions[row] : g;
    }
  }
}

struct CompactArgs {
  CacheView c;
  const int32_t *table, *len, *kept, *n_kept, *table_out;
  int width, width_out, kept_stride, tiles;
};

// One workgroup of 4 P threads makes one new page of one head of K or V.  Five trips to memory one after the other (counts,
// kept entry, table, codes and scale, then the writes): 6.6 us for 2048 of 32768 tokens of 8 heads, of which the 8.6 MB are 1.8.
template <int FMT>
__global__ void cache_compact(CompactArgs a) {
  __shared__ float part[16];
  const CacheView &c = a.c;
  int id = blockIdx.x;
  const bool is_v = id & 1;
  id >>= 1;
  const int head = id % c.H;
  id /= c.H;
  const int tile = id % a.tiles, b = id / a.tiles;
  const int total = min(min(a.n_kept[b], a.kept_stride), a.width_out * c.P);
  const int begin = tile * c.P;
  if (begin >= total) return;
  const int page = a.table_out[(size_t)b * a.width_out + tile];
  if (page < 0 || page >= c.n_pages) return;
  const int len = min(a.len[b], a.width * c.P);
  const int32_t *kept = a.kept + ((size_t)b * c.H + head) * a.kept_stride;
  const uint8_t *codes = is_v ? c.v : c.k;
  const float *scales = is_v ? c.vs : c.ks;
  const int across = threadIdx.x % kAcross, slot0 = threadIdx.x / kAcross * kQuad;
  u2 w[kQuad];
  float from[kQuad];
  int where[kQuad];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < kQuad; ++i) {
    const int g = begin + slot0 + i;
    const int t = g < total ? kept[g] : -1;
    w[i] = u2{0, 0};
    from[i] = kTinyScale;
    where[i] = -1;
    if (t >= 0 && t < len) {
      const int p = a.table[(size_t)b * a.width + t / c.P];
      if (p >= 0 && p < c.n_pages) {
        const size_t row = page_row(c, p, head) + t % c.P;
        w[i] = *reinterpret_cast<const u2 *>(codes + row * kHeadDim + across * kPer);
        from[i] = scales[(size_t)p * c.H + head];
        where[i] = c.pos ? c.pos[row] : t;
      }
    }
    amax = fmaxf(amax, Code<FMT>::magnitude(max(Code<FMT>::largest4(w[i][0]), Code<FMT>::largest4(w[i][1]))) * from[i]);
  }
  amax = block_max(amax, part);
  const float s = Code<FMT>::scale_for(fminf(amax, FLT_MAX));        // (127 times a rounded scale may lie above the largest number)
  const size_t row0 = page_row(c, page, head);
  uint8_t *out = (is_v ? c.v : c.k) + row0 * kHeadDim;
#pragma unroll
  for (int i = 0; i < kQuad; ++i) {
    *reinterpret_cast<u2 *>(out + (size_t)(slot0 + i) * kHeadDim + across * kPer) =
        u2{Code<FMT>::rescale4(w[i][0], from[i], s), Code<FMT>::rescale4(w[i][1], from[i], s)};
    if (c.pos && !is_v && across == 0) c.pos[row0 + slot0 + i] = where[i];
  }
  if (threadIdx.x == 0) (is_v ? c.vs : c.ks)[(size_t)page * c.H + head] = s;
}

// A workgroup copies one head's part of a page, K and V (96 pages of 64 tokens, 8 heads, 25 MB: 4.9 us).
__global__ __launch_bounds__(256) void cache_copy(CacheView c, const int32_t *pairs) {
  const int from = pairs[2 * (blockIdx.x / c.H)], to = pairs[2 * (blockIdx.x / c.H) + 1], head = blockIdx.x % c.H;
  if (from < 0 || from >= c.n_pages || to < 0 || to >= c.n_pages || from == to) return;
  const size_t src = page_row(c, from, head), dst = page_row(c, to, head);
  const u4 *k = reinterpret_cast<const u4 *>(c.k + src * kHeadDim), *v = reinterpret_cast<const u4 *>(c.v + src * kHeadDim);
  u4 *ko = reinterpret_cast<u4 *>(c.k + dst * kHeadDim), *vo = reinterpret_cast<u4 *>(c.v + dst * kHeadDim);
  for (int i = threadIdx.x; i < c.P * 8; i += 256) {
    const u4 x = k[i], y = v[i];
    ko[i] = x;
    vo[i] = y;
  }
  if (c.pos)
    for (int i = threadIdx.x; i < c.P; i += 256) c.pos[dst + i] = c.pos[src + i];
  if (threadIdx.x == 0) {
    c.ks[(size_t)to * c.H + head] = c.ks[(size_t)from * c.H + head];
    c.vs[(size_t)to * c.H + head] = c.vs[(size_t)from * c.H + head];
  }
}

template <int FMT>
void launch_append(const AppendArgs &a, int dtype, dim3 grid, dim3 block, hipStream_t st) {
  if (dtype == SPINDLE_F32) hipLaunchKernelGGL((cache_append<SPINDLE_F32, FMT>), grid, block, 0, st, a);
  else if (dtype == SPINDLE_F16) hipLaunchKernelGGL((cache_append<SPINDLE_F16, FMT>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((cache_append<SPINDLE_BF16, FMT>), grid, block, 0, st, a);
}

constexpr int64_t kMostBlocks = 1 << 22;        // a grid holds less than 2^32 threads, a block up to 1024

}  // namespace
}  // namespace spindle

using namespace spindle;

extern "C" spindle_status spindle_cache_append(const spindle_cache *cache, const int32_t *table, int32_t table_width,
                                               const int32_t *len, int32_t batch, const int32_t *cu_new, int32_t max_new,
                                               int32_t total_new, const void *K, const void *V, int32_t dtype, int64_t stride_b,
                                               int64_t stride_h, int64_t stride_t, const int32_t *positions, void *stream) {
  AppendArgs a{};
  if (spindle_status s = check_cache(cache, &a.c)) return s;
  if (spindle_status s = check_table(table, table_width, len, batch, a.c)) return s;
  if (dtype != SPINDLE_F32 && dtype != SPINDLE_F16 && dtype != SPINDLE_BF16) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (max_new < 0 || total_new < 0) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "max_new and total_new must be >= 0");
  if (!cu_new && (int64_t)batch * max_new != total_new)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "without cu_new every sequence gets max_new tokens: total_new must be batch * max_new");
  if (stride_b < 0 || stride_h < kHeadDim || stride_t < kHeadDim) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "strides must be >= 0, those of heads and tokens >= head_dim");
  if ((stride_b | stride_h | stride_t) & 7) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "strides must be multiples of 8 elements");
  if (max_new == 0 || total_new == 0) return SPINDLE_OK;            // (tensors without elements have no address)
  if (!K || !V) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "K and V are required");
  if ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  const int elt = dtype_bytes(dtype);
  a.table = table, a.len = len, a.cu = cu_new, a.positions = positions;
  a.K = static_cast<const char *>(K), a.V = static_cast<const char *>(V);
  a.sb = stride_b * elt, a.sh = stride_h * elt, a.st = stride_t * elt;
  a.width = table_width, a.max_new = max_new, a.total_new = total_new, a.rows = cu_new ? total_new : max_new;
  a.tiles = (int)(((int64_t)max_new + a.c.P - 2) / a.c.P + 1);
  if (a.tiles > table_width) a.tiles = table_width;
  const int64_t blocks = (int64_t)batch * a.tiles * a.c.H * 2;
  if (blocks >= kMostBlocks) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "too many pages in one call: split the batch");
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    ProfScope prof("cache_append", st);
    if (cache->format == SPINDLE_E4M3) launch_append<SPINDLE_E4M3>(a, dtype, dim3((unsigned)blocks), dim3(4 * a.c.P), st);
    else launch_append<SPINDLE_I8>(a, dtype, dim3((unsigned)blocks), dim3(4 * a.c.P), st);
  }
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}

extern "C" spindle_status spindle_cache_compact(const spindle_cache *cache, const int32_t *table, int32_t table_width,
                                                const int32_t *len, int32_t batch, const int32_t *kept_idx, int32_t kept_stride,
                                                const int32_t *n_kept, const int32_t *table_out, int32_t out_width, void *stream) {
  CompactArgs a{};
  if (spindle_status s = check_cache(cache, &a.c)) return s;
  if (spindle_status s = check_table(table, table_width, len, batch, a.c)) return s;
  if (spindle_status s = check_table(table_out, out_width, n_kept, batch, a.c)) return s;
  if (!kept_idx || kept_stride < 1) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "kept_idx is required and kept_stride must be >= 1");
  a.table = table, a.len = len, a.kept = kept_idx, a.n_kept = n_kept, a.table_out = table_out;
  a.width = table_width, a.width_out = out_width, a.kept_stride = kept_stride;
  a.tiles = (int)(((int64_t)kept_stride + a.c.P - 1) / a.c.P);
  if (a.tiles > out_width) a.tiles = out_width;
  const int64_t blocks = (int64_t)batch * a.tiles * a.c.H * 2;
  if (blocks >= kMostBlocks) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "too many pages in one call: split the batch");
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    ProfScope prof("cache_compact", st);
    if (cache->format == SPINDLE_E4M3) hipLaunchKernelGGL((cache_compact<SPINDLE_E4M3>), dim3((unsigned)blocks), dim3(4 * a.c.P), 0, st, a);
    else hipLaunchKernelGGL((cache_compact<SPINDLE_I8>), dim3((unsigned)blocks), dim3(4 * a.c.P), 0, st, a);
  }
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}

extern "C" spindle_status spindle_cache_copy(const spindle_cache *cache, const int32_t *pairs, int32_t n_pairs, void *stream) {
  CacheView c;
  if (spindle_status s = check_cache(cache, &c)) return s;
  if (n_pairs < 0) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "n_pairs must be >= 0");
  if (n_pairs == 0) return SPINDLE_OK;
  if (!pairs) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "pairs is required");
  if ((int64_t)n_pairs * c.H >= kMostBlocks) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "too many pages in one call: split the pairs");
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    ProfScope prof("cache_copy", st);
    hipLaunchKernelGGL(cache_copy, dim3((unsigned)(n_pairs * c.H)), dim3(256), 0, st, c, pairs);
  }
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}
