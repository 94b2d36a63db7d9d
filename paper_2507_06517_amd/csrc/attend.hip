// Attention over the paged cache in 8 bits: few query rows (decode steps, drafted tokens), and the calls.
#include "attend.h"

namespace spindle {
namespace {

constexpr int kTile = 32;                        // tokens of a step

// A step's tokens.  Its page (negative: absent) is looked up a step before its codes are asked for.
template <int kMode>
struct Tile {
  u4 k[4];                                       // [sub * 2 + h]: row 16 sub + lane % 16, bytes 64 h + 16 g ..
  u2 v[8];                                       // [4 a + i]: row 16 a + 4 g + i, bytes 8 (lane % 16) ..
  int pos[kMode == kBiased ? 8 : 1];
  float ks, vs;
  bool there;

  __device__ __forceinline__ void load(const CacheView &c, int page, int head, int t, int lane) {
    there = (uint32_t)page < (uint32_t)c.n_pages;
    if (!there) return;
    const int x = lane & 15, g = lane >> 4, slot = t & (c.P - 1);
    const uint32_t number = page_number(c, page, head), k_lane = x * kHeadDim + 16 * g, v_lane = 4 * g * kHeadDim + 8 * x;
    const uint64_t at = page_bytes(c, number, slot);
    const uint8_t *kp = c.k + at, *vp = c.v + at;
    ks = uniform_load_at(c.ks, number);
    vs = uniform_load_at(c.vs, number);
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int h = 0; h < 2; ++h) k[sub * 2 + h] = *reinterpret_cast<const u4 *>(kp + (k_lane + (16 * sub * kHeadDim + 64 * h)));
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * a + i] = *reinterpret_cast<const u2 *>(vp + (v_lane + (16 * a + i) * kHeadDim));
    if (kMode == kBiased) {
      if (c.pos) {
        const int32_t *const at_pos = c.pos + (((uint64_t)number << c.shift) + (uint32_t)slot);
        load_positions(at_pos + 4 * g, pos);
        load_positions(at_pos + 16 + 4 * g, pos + 4);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) pos[j] = t + (j >> 2) * 16 + 4 * g + (j & 3);
      }
    }
  }
  // Keeps the compiler from unpacking the codes where they are loaded, which would wait for them there (32 ragged sequences:
  // 115 us, and 39 held).
  __device__ __forceinline__ void hold_k() {
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(k[i]));
  }
  __device__ __forceinline__ void hold_v() {
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v[i]));
  }
};

// One workgroup attends 16 rows (tokens x query heads of one KV head) over one chunk of a sequence; its waves take
// tiles of 32 tokens in turn and are joined at the end.  S^T = K Q^T leaves a lane with the logits of one query row
// for tokens 4 g + i, which is where O^T = V^T P^T takes its weights from: the softmax stays in registers, and a row's
// statistics are found by two lane exchanges.  Codes go from memory to registers in 16-byte (K) and 8-byte (V) pieces of whole
// rows and never through LDS: a wave's 32 x 8 bytes of V are turned by 32 byte permutes, which the memory leaves time for.
//
// Bound by memory where contexts are long.  One token of 131071 (f16, E4M3, 268 MB): 42 us, 6.4 TB/s with part of it from the
// last-level cache, 4.6 with nothing cached (58 us with the join); a large copy reaches 4.9.  32 ragged sequences (bf16, integers,
// 136 MB): 35 us, of which a workgroup's start and end (three trips to memory, the join of the waves) are 5.  Four waves on a SIMD
// hide the trips better than two or three with a tile in flight ahead (35 and 39 us); two row tiles a wave share what is unpacked
// and were slower (drafted tokens 20 and 25 us).  1024 or 4096 workgroups instead of 2048: 62 and 42 against 39 us with the join.
// Short contexts are bound by the trips that wait for each other (drafted f32 tokens over 1000 to 2055: 19 us, vector
// instructions busy for 28 % of it, matrix instructions for 6: two steps a wave between those trips and the join).
// The biased forms have 4 to 7 registers more than four waves leave (f32: one more than three do), which spill: 32 ragged sequences
// with stored positions 46 us, 38 without; three waves a SIMD hold them and take 48.
template <int DT, int FMT, int kMode, int kWaves>
__global__ __launch_bounds__(kWaves * 64, DT == SPINDLE_F32 ? 3 : 4) void attend(AttendArgs a) {
  typedef typename Elem<DT>::type T;
  typedef Num<DT> N;
  typedef typename N::Q Q;
  const CacheView &c = a.c;
  const int lane = lane_id(), x = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // heads first, chunks last: neighbouring workgroups go to different dies, and the chunks that a short sequence lacks
  // come at the end for all of them
  int id = blockIdx.x;
  const int head = id % c.H;
  id /= c.H;
  const int row_tile = id % a.row_tiles;
  id /= a.row_tiles;
  const int b = id % a.batch, split = id / a.batch;
  // what the first tile's address hangs on is asked for at once
  const int begin = split * a.piece, first = begin + wave * kTile;
  const int32_t *table = a.table + (size_t)b * a.width;
  const int first_page = uniform_load(table + min(first >> c.shift, a.width - 1));
  const int len_b = uniform_load(a.len + b), cu0 = a.cu ? uniform_load(a.cu + b) : b * a.max_q, cu1 = a.cu ? uniform_load(a.cu + b + 1) : cu0 + a.max_q;
  const int prefix_b = a.prefix ? uniform_load(a.prefix + b) : 0;
  const int len = min(max(len_b, 0), a.width << c.shift), prefix = min(max(prefix_b, 0), len);
  const int t0 = cu0, m = min(max(cu1 - cu0, 0), a.max_q);
  const int rows = m * a.group, row_begin = row_tile * (kRows);
  const int first_q = len_b - m;                 // slot of the first new token
  if (row_begin >= rows || t0 < 0 || t0 > a.total_q - m || (begin >= len && split > 0)) return;
  // the rows are in the order of their tokens: the first sees least, the last most
  const int last_row = min(row_begin + kRows, rows) - 1;
  const int least = max(min(first_q + row_begin / a.group + 1, len), prefix);
  const int end = max(min(first_q + last_row / a.group + 1, len), prefix);
  auto page_at = [&](int t) { return t < end ? uniform_load_at(table, t >> c.shift) : -1; };
  Tile<kMode> tile;
  tile.load(c, first < end ? first_page : -1, head, first, lane);
  int page;

  RowState st;
  typename Q::frag q[4][N::kQ];
  {
    const int row = row_begin + x, i = row / a.group, hq = head * a.group + row % a.group;
    const bool on = row < rows;
    st.limit = on ? max(min(first_q + i + 1, len), prefix) : 0;
    st.m = -INFINITY;
    st.l = 0.f;
    st.slope = kMode == kBiased && a.slopes && on ? a.slopes[hq] * kLog2e : 0.f;
    st.q_at = kMode == kBiased && on ? (a.q_pos ? a.q_pos[t0 + i] : first_q + i) : 0;
    load_query<DT, 4>(q, a.Q + (size_t)(t0 + i) * a.qst + (size_t)hq * a.qsh, on, [g](int s) { return 64 * (s >> 1) + 16 * g + 8 * (s & 1); });
  }

  const float factor = kMode == kPlain ? a.scale * kLog2e : a.scale;
  f4 o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = f4{0, 0, 0, 0};

  auto step = [&](int t) {
    tile.hold_k();
    f4 s[2] = {f4{0, 0, 0, 0}, f4{0, 0, 0, 0}};
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const u4 w = tile.k[sub * 2 + (k >> 1)];
        const typename Q::frag kk = Q::template codes<FMT>(w[2 * (k & 1)], w[2 * (k & 1) + 1]);
#pragma unroll
        for (int part = N::kQ - 1; part >= 0; --part) s[sub] = Q::mma(kk, q[k][part], s[sub]);
      }
    const float f = fmaxf(factor * tile.ks, kTinyScale), slope = logit_slope<kMode>(f, a), offset = logit_offset<kMode>(a);
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = raw_logit<kMode>(s[j >> 2][j & 3], f, a, st, tile.pos[kMode == kBiased ? j : 0]);
    if (t + kTile > least) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (t + (j >> 2) * 16 + 4 * g + (j & 3) >= st.limit) w[j] = -INFINITY;
    }
    float top = w[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = larger(top, w[j]);
    bool scaled;
    const float back = gather(st, __builtin_fmaf(over_groups_max(top), slope, offset), &scaled);
    const float base = offset - (st.m == -INFINITY ? 0.f : st.m + kSlack);
    // V's scale goes into the weights, but for an E4M3 scale's power of two, which goes into the operands
    const float v_scale = FMT == SPINDLE_E4M3 ? operand_scale(tile.vs) : 1.f, v_rest = tile.vs * (1.f / v_scale);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(w[j], slope, base));
      st.l += w[j];
      w[j] *= v_rest;
    }
    Weights::frag p[N::kP];
    Weights::split<N::kP>(w, p);
    if (scaled) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= back;
    }
    tile.hold_v();
    if (t + kTile > len) {                                          // what lies behind the last token may be anything
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (t + (j >> 2) * 16 + 4 * g + (j & 3) >= len) tile.v[j] = u2{0, 0};
    }
    uint32_t col[2][8];                                             // [a][i]: dimension 8 x + i, tokens 16 a + 4 g + 0..3
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int lo = 0; lo < 2; ++lo)
        transpose4(tile.v[4 * h][lo], tile.v[4 * h + 1][lo], tile.v[4 * h + 2][lo], tile.v[4 * h + 3][lo], &col[h][4 * lo]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Weights::frag vv = Weights::codes<FMT>(col[0][i], col[1][i], v_scale);
#pragma unroll
      for (int part = N::kP - 1; part >= 0; --part) o[i] = Weights::mma(vv, p[part], o[i]);
    }
  };
  constexpr int kStride = kWaves * kTile;
  const int skip = (a.splits - 1) * a.piece;     // to the chunk's next piece
  auto after = [&](int t) { return t + kStride + (((t + kStride) & (a.piece - 1)) < kStride ? skip : 0); };
  for (int t = first, then; t < end; t = then) {
    if (t > first) tile.load(c, page, head, t, lane);
    then = after(t);
    page = page_at(then);
    if (tile.there) step(t);
  }

  // The waves' results, divided by their own sums, are joined: output row x, dimension 32 g + 8 e + i is o[i][e].
  __shared__ float so[kWaves][kRows][kHeadDim + 4];
  __shared__ float2 sml[kWaves][kRows];
  const float l = over_groups_sum(st.l);
  const float inv = l > 0.f ? 1.f / l : l;                          // a row that saw nothing: 0; NaN stays
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 8; ++i) so[wave][x][32 * g + 8 * e + i] = o[i][e] * inv;
  if (g == 0) sml[wave][x] = float2{st.m, l};
  __syncthreads();
  const int y = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;       // a thread takes 8 dimensions of a row
  const int row = row_begin + y;
  if (y >= kRows || row >= rows) return;
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sml[w][y].x);
  float sum = 0.f, weight[kWaves], res[8];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    weight[w] = sml[w][y].y == 0.f ? 0.f : sml[w][y].y * __builtin_amdgcn_exp2f(sml[w][y].x - top);
    sum += weight[w];
  }
  const float inv2 = sum > 0.f ? 1.f / sum : sum;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += weight[w] * so[w][y][d + j];
    res[j] = v * inv2;
  }
  const size_t at = (size_t)(t0 + row / a.group) * a.heads_q + head * a.group + row % a.group;
  if (a.splits == 1) {
    T e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = Elem<DT>::from_float(res[j]);
    __builtin_memcpy(__builtin_assume_aligned(a.out + (at * kHeadDim + d) * sizeof(T), 16), e, sizeof(e));
    if (a.lse && d == 0) a.lse[at] = lse_of(top, sum);
  } else {
    float *po = a.part_o + (at * a.splits + split) * kHeadDim + d;
    *reinterpret_cast<f4 *>(po) = f4{res[0], res[1], res[2], res[3]};
    *reinterpret_cast<f4 *>(po + 4) = f4{res[4], res[5], res[6], res[7]};
    if (d == 0) a.part_ml[at * a.splits + split] = float2{top, sum};
  }
}

// Joins the chunks of a row: a workgroup per row.  Sixteen groups of 32 threads (4 dimensions each) take every sixteenth
// chunk, so that a row of 256 chunks is 16 steps and not 256.
constexpr int kJoinGroups = 16, kJoinChunks = 32 * kJoinGroups;
template <int DT>
__global__ __launch_bounds__(32 * kJoinGroups) void attend_join(AttendArgs a) {
  const int b = blockIdx.x / a.max_q, i = blockIdx.x % a.max_q, hq = blockIdx.y;
  const int t0 = a.cu ? a.cu[b] : b * a.max_q;
  const int m = a.cu ? min(max(a.cu[b + 1] - t0, 0), a.max_q) : a.max_q;
  if (i >= m || t0 < 0 || t0 > a.total_q - m) return;
  const size_t at = (size_t)(t0 + i) * a.heads_q + hq;
  const int d = threadIdx.x & 31, group = threadIdx.x >> 5;
  const float2 *ml = a.part_ml + at * a.splits;
  const f4 *po = reinterpret_cast<const f4 *>(a.part_o + at * a.splits * kHeadDim) + d;
  const int len = min(max(a.len[b], 0), a.width * a.c.P), n = min((len + a.piece - 1) / a.piece, a.splits);
  // the weights by all threads at once, then the sums: two trips to memory for a row of up to 512 chunks
  __shared__ float weight[kJoinChunks], part[kJoinGroups];
  float top = -INFINITY, sum = 0.f;
  f4 v = {0, 0, 0, 0};
  for (int s0 = 0; s0 < n; s0 += kJoinChunks) {
    const int s1 = s0 + (int)threadIdx.x;
    const float2 mine = s1 < n ? ml[s1] : float2{-INFINITY, 0.f};
    float most = mine.x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
    if (s0) __syncthreads();
    if (d == 0) part[group] = most;
    __syncthreads();
    const float was = top;
#pragma unroll
    for (int k = 0; k < kJoinGroups; ++k) top = fmaxf(top, part[k]);
    weight[threadIdx.x] = mine.y == 0.f ? 0.f : mine.y * __builtin_amdgcn_exp2f(mine.x - top);
    __syncthreads();
    const float back = was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(was - top);
    sum *= back;
    v *= back;
    const int m1 = min(n - s0, kJoinChunks);
#pragma unroll 8
    for (int s = group; s < m1; s += kJoinGroups) {
      const f4 x = po[(size_t)(s0 + s) * 32];
      sum += weight[s];
      v += weight[s] * x;
    }
  }
  __shared__ f4 sv[kJoinGroups][32];
  __shared__ float ss[kJoinGroups];
  sv[group][d] = v;
  if (d == 0) ss[group] = sum;
  __syncthreads();
  if (group) return;
#pragma unroll
  for (int k = 1; k < kJoinGroups; ++k) {
    v += sv[k][d];
    sum += ss[k];
  }
  const float inv = sum > 0.f ? 1.f / sum : sum;                    // 0 for a row that sees nothing, NaN stays
  typename Elem<DT>::type *out = reinterpret_cast<typename Elem<DT>::type *>(a.out) + at * kHeadDim + 4 * d;
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = Elem<DT>::from_float(v[j] * inv);
  if (a.lse && d == 0) a.lse[at] = lse_of(top, sum);
}

// The same for rows of few chunks: 32 threads per row, sixteen rows to a workgroup.
template <int DT>
__global__ __launch_bounds__(32 * kJoinGroups) void attend_join_few(AttendArgs a) {
  const long long id = (long long)blockIdx.x * kJoinGroups + (threadIdx.x >> 5);
  const int hq = (int)(id % a.heads_q), b = (int)(id / a.heads_q / a.max_q), i = (int)(id / a.heads_q % a.max_q), d = threadIdx.x & 31;
  if (b >= a.batch) return;
  const int t0 = a.cu ? a.cu[b] : b * a.max_q;
  const int m = a.cu ? min(max(a.cu[b + 1] - t0, 0), a.max_q) : a.max_q;
  if (i >= m || t0 < 0 || t0 > a.total_q - m) return;
  const size_t at = (size_t)(t0 + i) * a.heads_q + hq;
  const float2 *ml = a.part_ml + at * a.splits;
  const f4 *po = reinterpret_cast<const f4 *>(a.part_o + at * a.splits * kHeadDim) + d;
  constexpr int kAtOnce = 8;
  const int len = min(max(a.len[b], 0), a.width << a.c.shift), n = min((len + a.piece - 1) / a.piece, a.splits);
  float top = -INFINITY, sum = 0.f;
  f4 v = {0, 0, 0, 0};
  for (int s0 = 0; s0 < n; s0 += kAtOnce) {      // that many chunks' loads in flight
    float2 w[kAtOnce];
    f4 x[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int s = min(s0 + k, n - 1);
      w[k] = ml[s];
      x[k] = po[s * 32];
    }
    const float was = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, s0 + k < n ? w[k].x : -INFINITY);
    const float back = was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(was - top);
    sum *= back;
    v *= back;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float weight = s0 + k < n && w[k].y != 0.f ? w[k].y * __builtin_amdgcn_exp2f(w[k].x - top) : 0.f;
      sum += weight;
      v += weight * x[k];
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : sum;                    // 0 for a row that sees nothing, NaN stays
  typename Elem<DT>::type e[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) e[j] = Elem<DT>::from_float(v[j] * inv);
  __builtin_memcpy(__builtin_assume_aligned(reinterpret_cast<typename Elem<DT>::type *>(a.out) + at * kHeadDim + 4 * d, 8), e, sizeof(e));
  if (a.lse && d == 0) a.lse[at] = lse_of(top, sum);
}

// Waves of a workgroup: many where one workgroup takes a whole context, without a second kernel.
constexpr int kFewWaves = 4, kManyWaves = 8, kTarget = 2048;

// Many waves pay while the workgroups all run at once, two on a compute unit and one of f32, which has more registers (f16, bf16
// integers and f32, contexts of 300: 256 workgroups 12.1, 11.4 and 11.1 us and few waves 16.3, 16.3 and 15.5; 800: 17.9, 22.3
// and 27.4 us and 15.9, 18.5 and 19.3), and until the chunks of few waves make up for the launch of their join: 8 workgroups with
// contexts of 1000 11.3, 13.3 and 13.3 us (15.7, 15.6 and 15.5), of 2000 15.9, 19.7 and 19.1 (16.1, 15.9 and 15.5); with 160
// workgroups, which leave the chunks less of the chip, of 2000 18.0, 22.4 and 21.9 us (21.5, 23.3 and 23.2).
bool many_waves(int64_t units, int64_t tokens, int dtype) {
  return units <= (dtype == SPINDLE_F32 ? 256 : 512) && tokens <= (units < 128 ? 1280 : 2048);
}

struct Plan {
  bool rows;                                     // the kernel for many rows
  int waves, row_tiles, splits, piece;           // tokens of a piece: a power of two
  size_t bytes;
};

// How the work is cut: rows in tiles, tokens in pieces that go to the chunks in turn, so that the cut, which knows the table's
// width and not the lengths, leaves every chunk its share of a sequence of any length; chunks enough to give the chip even work.
Plan plan_attend(const CacheView &c, int batch, int width, int max_q, int total_q, int group, int dtype) {
  Plan p;
  const int64_t rows = (int64_t)max_q * group, tokens = (int64_t)width * c.P;
  int64_t splits = 1;
  // Rows of 16-bit queries share unpacked tokens from the fifth 16-row tile on (6 x 8 heads, f16, integers, 2000 tokens: 64 rows
  // 28 us here and 31 there, 128 rows 38 and 36, 256 rows 56 and 47).
  p.rows = rows > 64 && dtype != SPINDLE_F32;
  if (p.rows) {
    // What a cut takes, in microseconds: a step of 64 tokens 1.9 while every compute unit has one workgroup, 3 with two, which is
    // as many as it runs at a time; 6 to begin and to end; the join's kernel 5, and its bytes written and read at 4 TB/s.
    // No more than two rounds of workgroups: the table may be far wider than its sequences (five prompts of up to 1500 in one of
    // 131072 tokens: 117 us with as many as the width asks for, 62 with these).
    p.row_tiles = (int)((rows + kManyRows - 1) / kManyRows);
    const int64_t units = (int64_t)batch * c.H * p.row_tiles;
    p.piece = kManyStep;
    double best = 1e30;
    for (int64_t s = 1; s <= 64 && (s == 1 || ((s - 1) * kManyStep < tokens && units * s <= 1024)); ++s) {
      const int64_t n = units * s, steps = (tokens + 64 * s - 1) / (64 * s);
      const double t = (n <= 256 ? (double)steps * 1.9 + 6 : (double)((n + 511) / 512) * ((double)steps * 3.0 + 6)) +
                       (s > 1 ? 5 + (double)n * kManyRows * kHeadDim * 8 / 4e6 : 0);
      if (t < best) best = t, splits = s;
    }
  } else {
    p.row_tiles = (int)((rows + kRows - 1) / kRows);
    const int64_t units = (int64_t)batch * c.H * p.row_tiles;
    p.waves = rows <= kRows && many_waves(units, tokens, dtype) ? kManyWaves : kFewWaves;
    p.piece = p.waves * kTile;
    const int64_t most = (tokens + p.piece - 1) / p.piece;
    splits = p.waves == kManyWaves ? 1 : kTarget / units;
    if (splits > most) splits = most;
    // a workgroup takes as long to begin and to end as for two steps, so chunks get up to four steps of each wave while
    // there are two workgroups for every compute unit
    while (splits > 1 && splits * 4 > most && units * splits >= 1024) splits = (splits + 1) / 2;
    if (splits < 1) splits = 1;
    // Pieces of up to eight steps, while they are as even over the chunks: then a short sequence among long ones has few
    // workgroups with much to do each (32 ragged sequences of up to 8192: pieces of one step 42 us, of eight 39).  One piece a
    // chunk would leave most of them without work where the table has room for far more than the sequences have (the same
    // in a table of 131072 tokens: 91 us and 42).
    const int64_t each = (most + splits - 1) / splits;
    for (int64_t n = 2; n <= 8 && (most + n * splits - 1) / (n * splits) * n <= each + each / 8; n *= 2) p.piece = (int)(p.waves * kTile * n);
  }
  // as few chunks as have no more pieces than with `splits`
  const int64_t all = (tokens + p.piece - 1) / p.piece, each = (all + splits - 1) / splits;
  p.splits = (int)((all + each - 1) / each);
  p.bytes = p.splits > 1 ? align_up((size_t)total_q * c.H * group * p.splits * kHeadDim * 4, 256) +
                               align_up((size_t)total_q * c.H * group * p.splits * sizeof(float2), 256)
                         : 0;
  return p;
}

template <int DT, int FMT, int kWaves>
void launch_waves(const AttendArgs &a, int mode, dim3 grid, hipStream_t st) {
  if (mode == kPlain) hipLaunchKernelGGL((attend<DT, FMT, kPlain, kWaves>), grid, dim3(kWaves * 64), 0, st, a);
  else if (mode == kCapped) hipLaunchKernelGGL((attend<DT, FMT, kCapped, kWaves>), grid, dim3(kWaves * 64), 0, st, a);
  else hipLaunchKernelGGL((attend<DT, FMT, kBiased, kWaves>), grid, dim3(kWaves * 64), 0, st, a);
}

template <int DT, int FMT>
void launch_attend(const AttendArgs &a, const Plan &p, int mode, dim3 grid, hipStream_t st) {
  if (p.waves == kManyWaves) launch_waves<DT, FMT, kManyWaves>(a, mode, grid, st);
  else launch_waves<DT, FMT, kFewWaves>(a, mode, grid, st);
}

template <int DT>
spindle_status launch_type(const AttendArgs &a, int fmt, const Plan &p, int mode, dim3 grid, hipStream_t st) {
  if (p.rows) {
    ProfScope prof("attend_rows", st);
    if (spindle_status s = launch_attend_rows(a, DT, fmt, mode, grid.x, st)) return s;
  } else {
    ProfScope prof("attend", st);
    if (fmt == SPINDLE_E4M3) launch_attend<DT, SPINDLE_E4M3>(a, p, mode, grid, st);
    else launch_attend<DT, SPINDLE_I8>(a, p, mode, grid, st);
  }
  if (a.splits > 1) {
    ProfScope prof("attend_join", st);
    // 32 threads a row are 2 us sooner with 1024 rows of 8 chunks (and 140 us with 120000 of 2); a whole workgroup has the
    // 256 chunks of 32 rows in half the time
    const int64_t rows = (int64_t)a.batch * a.max_q * a.heads_q;
    if (a.splits <= 16 || rows > 1024)
      hipLaunchKernelGGL((attend_join_few<DT>), dim3((unsigned)((rows + kJoinGroups - 1) / kJoinGroups)), dim3(32 * kJoinGroups), 0, st, a);
    else
      hipLaunchKernelGGL((attend_join<DT>), dim3((unsigned)(a.batch * a.max_q), (unsigned)a.heads_q), dim3(32 * kJoinGroups), 0, st, a);
  }
  return SPINDLE_OK;
}

spindle_status check_queries(int32_t batch, int32_t max_q, int32_t total_q, int32_t group, const CacheView &c, const void *cu) {
  if (max_q < 0 || total_q < 0) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "max_q and total_q must be >= 0");
  if (!cu && (int64_t)batch * max_q != total_q)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "without cu_q every sequence has max_q queries: total_q must be batch * max_q");
  if (group < 1) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "group_size must be >= 1");
  if (group > 256 || (int64_t)group * c.H > 65535) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "at most 256 query heads per KV head and 65535 in all");
  if ((int64_t)max_q * group > (1 << 30) || (int64_t)batch * max_q > (1 << 24))
    SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "too many queries in one call");
  return SPINDLE_OK;
}

}  // namespace
}  // namespace spindle

using namespace spindle;

extern "C" spindle_status spindle_attend_workspace_bytes(const spindle_cache *cache, int32_t batch, int32_t table_width, int32_t max_q,
                                                         int32_t total_q, int32_t group_size, int32_t dtype, size_t *bytes) {
  CacheView c;
  if (!bytes) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "bytes is NULL");
  if (spindle_status s = check_cache(cache, &c)) return s;
  if (spindle_status s = check_table(cache, table_width, cache, batch, c)) return s;
  if (spindle_status s = check_queries(batch, max_q, total_q, group_size, c, cache)) return s;
  if (dtype != SPINDLE_F32 && dtype != SPINDLE_F16 && dtype != SPINDLE_BF16) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  *bytes = max_q && total_q ? plan_attend(c, batch, table_width, max_q, total_q, group_size, dtype).bytes : 0;
  return SPINDLE_OK;
}

extern "C" spindle_status spindle_cache_attend(const spindle_cache *cache, const int32_t *table, int32_t table_width, const int32_t *len,
                                               int32_t batch, const int32_t *cu_q, int32_t max_q, int32_t total_q, const void *Q, int32_t dtype,
                                               int32_t group_size, int64_t stride_t, int64_t stride_h, float scale, float softcap,
                                               const float *slopes, const int32_t *prefix, const int32_t *q_pos, void *out, float *lse,
                                               void *workspace, size_t workspace_bytes, void *stream) {
  AttendArgs a{};
  if (spindle_status s = check_cache(cache, &a.c)) return s;
  if (spindle_status s = check_table(table, table_width, len, batch, a.c)) return s;
  if (spindle_status s = check_queries(batch, max_q, total_q, group_size, a.c, cu_q)) return s;
  if (dtype != SPINDLE_F32 && dtype != SPINDLE_F16 && dtype != SPINDLE_BF16) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (stride_t < kHeadDim || stride_h < kHeadDim || ((stride_t | stride_h) & 7))
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "strides must be >= head_dim and multiples of 8 elements");
  if (!(scale > 0.f) || !(scale < INFINITY)) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (!(softcap >= 0.f) || !(softcap < INFINITY)) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "softcap must be finite and >= 0 (0 = none)");
  if (max_q == 0 || total_q == 0) return SPINDLE_OK;                // (tensors without elements have no address)
  if (!Q || !out) SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "Q and out are required");
  if ((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(out)) & 15)
    SPINDLE_FAIL(SPINDLE_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  const Plan p = plan_attend(a.c, batch, table_width, max_q, total_q, group_size, dtype);
  if (p.bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < p.bytes))
    SPINDLE_FAIL(SPINDLE_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than %zu bytes", p.bytes);
  const int64_t blocks = (int64_t)batch * a.c.H * p.row_tiles * p.splits;
  if (blocks >= (1 << 23)) SPINDLE_FAIL(SPINDLE_ERR_UNSUPPORTED, "too many queries in one call");
  const int elt = dtype_bytes(dtype);
  a.table = table, a.len = len, a.cu = cu_q, a.prefix = prefix, a.q_pos = q_pos, a.slopes = slopes;
  a.Q = static_cast<const char *>(Q), a.out = static_cast<char *>(out), a.lse = lse;
  a.qst = stride_t * elt, a.qsh = stride_h * elt;
  // (a cap of less than 1e-30 makes logits of less than that, as 1e-30 does, whose inverse is a number)
  a.scale = scale, a.softcap = softcap > 0.f ? fmaxf(softcap, 1e-30f) : 0.f;
  a.cap_in = 2.f * kLog2e / a.softcap, a.cap_out = a.softcap * kLog2e, a.per_cap = 1.f / a.softcap;
  a.width = table_width, a.max_q = max_q, a.total_q = total_q, a.group = group_size, a.heads_q = a.c.H * group_size;
  a.batch = batch, a.splits = p.splits, a.piece = p.piece, a.row_tiles = p.row_tiles;
  if (p.bytes) {
    Carver w(workspace);
    a.part_o = w.take<float>((size_t)total_q * a.heads_q * p.splits * kHeadDim);
    a.part_ml = w.take<float2>((size_t)total_q * a.heads_q * p.splits);
  }
  const int mode = slopes || a.c.pos || softcap > kWideCap ? kBiased : softcap > 0.f ? kCapped : kPlain;
  const dim3 grid((unsigned)blocks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (spindle_status s = dtype == SPINDLE_F32 ? launch_type<SPINDLE_F32>(a, cache->format, p, mode, grid, st)
                         : dtype == SPINDLE_F16 ? launch_type<SPINDLE_F16>(a, cache->format, p, mode, grid, st)
                                                : launch_type<SPINDLE_BF16>(a, cache->format, p, mode, grid, st))
    return s;
  SPINDLE_HIP(hipGetLastError());
  return SPINDLE_OK;
}
