// Bookkeeping of the paged cache: which sequence holds which pages.  refs[p] counts the table entries that hold page p;
// a page is free when nothing holds it, and the free page of the lowest number is handed out first, so that the same calls
// give the same tables whatever order the workgroups run in.
#include "cache.h"

namespace spindle {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int held_pages(int len, int width, int shift) {
  return len > 0 ? min((int)(((unsigned)len + (1u << shift) - 1) >> shift), width) : 0;
}

// A workgroup per row: it takes its parent's pages (96 rows of up to 141 pages: 3.1 us, three trips to memory).
__global__ __launch_bounds__(kThreads) void pages_share(int32_t *refs, int n_pages, const int32_t *table, const int32_t *len, int rows_in,
                                                        int width, const int32_t *parent, int32_t *table_out, int32_t *len_out, int shift) {
  const int r = blockIdx.x, p = parent[r];
  const bool has = p >= 0 && p < rows_in;
  const int n = has ? len[p] : 0, held = held_pages(n, width, shift);
  for (int j = threadIdx.x; j < width; j += kThreads) {
    const int page = j < held ? table[(size_t)p * width + j] : -1;
    table_out[(size_t)r * width + j] = page;
    if (page >= 0 && page < n_pages) atomicAdd(&refs[page], 1);
  }
  if (threadIdx.x == 0) len_out[r] = n;
}

__global__ __launch_bounds__(kThreads) void pages_release(int32_t *refs, int n_pages, const int32_t *table, const int32_t *len, int width, int shift) {
  const int r = blockIdx.x, held = held_pages(len[r], width, shift);
  for (int j = threadIdx.x; j < held; j += kThreads) {
    const int page = table[(size_t)r * width + j];
    if (page >= 0 && page < n_pages) atomicSub(&refs[page], 1);
  }
}

constexpr int kReserveThreads = 1024, kMostRows = 4096, kMostWidth = 1 << 20, kEach = 16, kNear = 4096;   // pages that a thread looks at in one go

// Exclusive sum over the block's threads in their order, and the sum of all.
__device__ __forceinline__ int block_before(int v, int *shared, int *total) {
  const int wave = threadIdx.x >> 6, upto = lanes_up_to(v);
  __syncthreads();
  if (lane_id() == 63) shared[wave] = upto;
  __syncthreads();
  const int w = lane_id() < kReserveThreads / 64 ? shared[lane_id()] : 0;
  const int sums = lanes_up_to(w);
  *total = __shfl(sums, kReserveThreads / 64 - 1);
  return upto - v + (wave ? __shfl(sums, wave - 1) : 0);
}

// One workgroup does it all: what each row needs, a sum over the rows, the free pages in order, the new entries.  The time is
// that of trips to memory that wait for each other, not of the bytes (4.4 us for 4 rows, 11 for 96 that share 24 pages), so
// lengths, last pages and their counts are kept, and the counts of the first 16384 pages are asked for before anything else.
__global__ __launch_bounds__(kReserveThreads) void pages_reserve(int32_t *refs, int n_pages, int32_t *table, const int32_t *len,
                                                                 const int32_t *grow, int rows, int width, int shift, int32_t *len_out,
                                                                 int32_t *copies, int32_t *status, int32_t *free_list) {
  __shared__ __align__(16) int last_of[kMostRows];          // the half-full page that the row would write to
  __shared__ int begin_of[kMostRows], need_of[kMostRows], len_of[kMostRows], grow_of[kMostRows];   // need: new entries << 1 | the last page is copied
  __shared__ int near_list[kNear];                         // the first free pages; a call that takes more has the others in the workspace
  __shared__ int part[kReserveThreads / 64], too_narrow;
  const int tid = threadIdx.x, mask = (1 << shift) - 1;
  auto free_bits = [&](int p0) {                            // of the 16 pages of this thread
    const int p = p0 + tid * kEach;
    uint32_t bits = 0;
    if (p + kEach <= n_pages) {
      u4 r[kEach / 4];
#pragma unroll
      for (int i = 0; i < kEach / 4; ++i) __builtin_memcpy(&r[i], refs + p + 4 * i, 16);
#pragma unroll
      for (int i = 0; i < kEach; ++i) bits |= (r[i >> 2][i & 3] == 0 ? 1u : 0u) << i;
    } else {
      for (int i = 0; p + i < n_pages; ++i) bits |= (refs[p + i] == 0 ? 1u : 0u) << i;
    }
    return bits;
  };
  uint32_t is_free = free_bits(0);
  if (tid == 0) too_narrow = 0;
  int shared_by[kMostRows / kReserveThreads];
#pragma unroll
  for (int k = 0; k < kMostRows / kReserveThreads; ++k) {
    const int r = k * kReserveThreads + tid;
    shared_by[k] = 0;
    if (r >= rows) continue;
    const int n = max(len[r], 0), m = max(grow[r], 0), last = (n - 1) >> shift;
    int page = -1;
    if (m > 0 && (n & mask) != 0 && last < width) page = table[(size_t)r * width + last];
    if (page < 0 || page >= n_pages) page = -1;
    if (page >= 0) shared_by[k] = refs[page];
    last_of[r] = page;
    len_of[r] = n;
    grow_of[r] = m;
  }
  __syncthreads();
  int narrow = 0;
  long long need = 0;
#pragma unroll
  for (int k = 0; k < kMostRows / kReserveThreads; ++k) {
    const int r = k * kReserveThreads + tid;
    if (k * kReserveThreads >= rows) break;
    int mine = 0;
    if (r < rows) {
      const int n = len_of[r], page = last_of[r];
      const long long after = ((long long)n + grow_of[r] + mask) >> shift;
      int moves = 0;
      if (shared_by[k] > 1) {                               // the rows in their order: each that finds the page shared takes a copy
        int rank = 0;
        for (int q = 0; q < r && rank < shared_by[k] - 1; q += 4) {
          const int4 l = *reinterpret_cast<const int4 *>(&last_of[q]);
          rank += (l.x == page) + (q + 1 < r && l.y == page) + (q + 2 < r && l.z == page) + (q + 3 < r && l.w == page);
        }
        moves = rank < shared_by[k] - 1;
      }
      if (after > width) ++narrow;
      const long long fresh = min(after - (((long long)n + mask) >> shift), (long long)kMostWidth);
      mine = (int)fresh + moves;
      need_of[r] = mine << 1 | moves;
    }
    int total;
    const int before = block_before(mine, part, &total);
    if (r < rows) begin_of[r] = (int)need + before;         // only read when all fit
    need += total;
  }
  if (narrow) atomicAdd(&too_narrow, narrow);
  __syncthreads();
  // free pages in order, as many as are needed
  int found = 0;
  for (int p0 = 0; p0 < n_pages && found < need; p0 += kReserveThreads * kEach) {
    if (p0) is_free = free_bits(p0);
    int total;
    int at = found + block_before(__popc(is_free), part, &total);
    for (uint32_t m = is_free; m; m &= m - 1, ++at)
      if (at < need) (at < kNear ? near_list : free_list)[at] = p0 + tid * kEach + __ffs(m) - 1;
    found += total;
  }
  const int lacking = (int)min(max(need - found, 0ll), (long long)INT32_MAX);
  const bool fine = lacking == 0 && too_narrow == 0;
  __syncthreads();                                          // the list is written; every count was read
  for (int r = tid >> 6; r < rows; r += kReserveThreads / 64) {
    const int n = len_of[r], moves = need_of[r] & 1, count = need_of[r] >> 1, begin = begin_of[r];
    const int first = ((n + mask) >> shift) - moves;
    if (fine)
      for (int k = lane_id(); k < count; k += 64) {
        const int page = (begin + k < kNear ? near_list : free_list)[begin + k];
        table[(size_t)r * width + first + k] = page;
        refs[page] = 1;
        if (moves && k == 0) copies[2 * r + 1] = page;
      }
    if (lane_id() == 0) {
      len_out[r] = fine ? n + grow_of[r] : n;
      const bool moved = fine && moves;
      copies[2 * r] = moved ? last_of[r] : -1;
      if (!moved) copies[2 * r + 1] = -1;
      if (moved) atomicSub(&refs[last_of[r]], 1);
    }
  }
  if (tid == 0) {
    status[0] = lacking;
    status[1] = too_narrow;
  }
}

spindle_status check_pages(const void *refs, int32_t n_pages, const void *table, int32_t width, const void *len, int32_t rows,
                           int32_t page_tokens, int *shift) {
  if (!refs || !table || !len) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "refs, table and len are required");
  if (n_pages < 1 || width < 1 || rows < 1) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "n_pages, the table's width and its rows must be >= 1");
  if (n_pages >= (1 << 30)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "n_pages must be below 2^30");
  if (page_tokens != 32 && page_tokens != 64 && page_tokens != 128 && page_tokens != 256)
    SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "page_tokens must be 32, 64, 128 or 256, got %d", page_tokens);
  if ((int64_t)width * page_tokens > (1 << 30)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "a table's row may hold at most 2^30 tokens");
  if (width > kMostWidth) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "a table's row may hold at most %d pages", kMostWidth);
  if (rows > (1 << 22)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "too many rows");
  *shift = __builtin_ctz((unsigned)page_tokens);
  return SPINDLE_OK;
}

}  // namespace
}  // namespace spindle

using namespace spindle;

extern "C" spindle_status spindle_pages_share(int32_t *refs, int32_t n_pages, const int32_t *table, const int32_t *len, int32_t rows_in,
                                              int32_t table_width, int32_t page_tokens, const int32_t *parent, int32_t rows_out,
                                              int32_t *table_out, int32_t *len_out, void *stream) {
  int shift;
  if (spindle_status s = check_pages(refs, n_pages, table, table_width, len, rows_in, page_tokens, &shift)) return s;
  if (spindle_status s = check_pages(refs, n_pages, table_out, table_width, len_out, rows_out, page_tokens, &shift)) return s;
  if (!parent) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "parent is required");
  if (table == table_out || len == len_out) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "table_out and len_out must not be table and len");
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    ProfScope prof("pages_share", st);
    hipLaunchKernelGGL(pages_share, dim3((unsigned)rows_out), dim3(kThreads), 0, st, refs, n_pages, table, len, rows_in, table_width,
                       parent, table_out, len_out, shift);
  }
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}

extern "C" spindle_status spindle_pages_release(int32_t *refs, int32_t n_pages, const int32_t *table, const int32_t *len, int32_t rows,
                                                int32_t table_width, int32_t page_tokens, void *stream) {
  int shift;
  if (spindle_status s = check_pages(refs, n_pages, table, table_width, len, rows, page_tokens, &shift)) return s;
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    ProfScope prof("pages_release", st);
    hipLaunchKernelGGL(pages_release, dim3((unsigned)rows), dim3(kThreads), 0, st, refs, n_pages, table, len, table_width, shift);
  }
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}

extern "C" spindle_status spindle_pages_workspace_bytes(int32_t n_pages, size_t *bytes) {
  if (!bytes) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "bytes is NULL");
  if (n_pages < 1) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "n_pages must be >= 1");
  if (n_pages >= (1 << 30)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "n_pages must be below 2^30");
  *bytes = align_up((size_t)n_pages * 4, 256);
  return SPINDLE_OK;
}

extern "C" spindle_status spindle_pages_reserve(int32_t *refs, int32_t n_pages, int32_t *table, const int32_t *len, const int32_t *grow,
                                                int32_t rows, int32_t table_width, int32_t page_tokens, int32_t *len_out, int32_t *copies,
                                                int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
  int shift;
  if (spindle_status s = check_pages(refs, n_pages, table, table_width, len, rows, page_tokens, &shift)) return s;
  if (!grow || !len_out || !copies || !status) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "grow, len_out, copies and status are required");
  if (len == len_out) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "len_out must not be len");
  if (rows > kMostRows) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "at most %d rows in one call, got %d", kMostRows, rows);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < (size_t)n_pages * 4)
    SPINDLE_FAIL(SPINDLE_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than %zu bytes", (size_t)n_pages * 4);
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    ProfScope prof("pages_reserve", st);
    hipLaunchKernelGGL(pages_reserve, dim3(1), dim3(kReserveThreads), 0, st, refs, n_pages, table, len, grow, rows, table_width, shift,
                       len_out, copies, status, static_cast<int32_t *>(workspace));
  }
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}
