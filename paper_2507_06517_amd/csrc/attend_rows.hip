// Attention over the paged cache in 8 bits: many query rows (pieces of prompts, whole prompts).
#include "attend.h"

namespace spindle {
namespace {

constexpr int kStep = kManyStep;                 // tokens of a step
constexpr int kThreads = 256;
constexpr int kFrag = 1024;                      // bytes of an operand of one wave
constexpr int kBuffer = 16 * kFrag;              // K or V of a step as operands

// One workgroup attends 128 rows over one chunk: a wave has 32 rows of its own, and all four share the step's tokens.
// Codes become operands once for all of them, on their way into LDS, in the order in which the matrix instructions
// take them (V is turned on the way); a wave would otherwise spend as many vector instructions on unpacking as on the
// softmax of its rows.  Two buffers: while one step is computed the next one is unpacked and the one after it is on its way,
// with one barrier a step.  Two workgroups share a compute unit, so that one's products run beside the other's softmax.
//
// Bound by the matrix and vector instructions together, and by the clock that falls with them: 2048 bf16 queries of 4 x 8 heads
// over 16 Ki tokens take 0.71 to 0.79 ms, 0.60 with operands of zeros.  The products are 0.515 TFLOP, 0.43 ms at what a library
// product of 8192^3 reaches here (1.2 PFLOP/s), and 0.77 TFLOP with the second bf16 half of the weights, 0.64 ms.  Matrix
// instructions are busy for 49 % of the cycles, vector instructions for 54.  Tried, at 0.80 for this form: eight waves of which four
// are half a step behind (0.77, but 90 us against 73 for five short f16 prompts with capped scores), eight in step (0.80, 97),
// 16x16 products (0.79), V's products a step late (0.87), raised wave priority for products (0.86), forced interleaving (0.81).
// Slopes and stored positions add vector instructions: the same 2048 queries 1.05 ms (1.13 with one loop for stored and plain
// positions, whose registers spill; 1.20 with a load for each position).  Short prompts are bound by the chain of the longest row
// tile: five f16 prompts of 200 to 1500 tokens with capped scores take 66 us, in which 400 workgroups of up to 24 steps run all at
// once and no unit is busy (vector instructions 28 %, matrix instructions 13, LDS 11).
template <int DT, int FMT, int kMode>
__global__ __launch_bounds__(kThreads, 2) void attend_rows(AttendArgs a) {
  typedef typename Elem<DT>::type T;
  typedef Num<DT> N;
  typedef typename N::Q Q;
  typedef Weights::frag frag;
  extern __shared__ char lds[];                  // [2][K: half 2 x step 8][64 lanes][16 bytes], [2][V: step 4 x tile 4][64][16]
  const CacheView &c = a.c;
  const int tid = threadIdx.x, lane = lane_id(), x = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // heads first: the workgroups of one head, which read the same tokens, go to the same die where there are 8 heads; the last
  // rows first: they see most
  int id = blockIdx.x;
  const int head = id % c.H;
  id /= c.H;
  const int row_tile = a.row_tiles - 1 - id % a.row_tiles;
  id /= a.row_tiles;
  const int b = id % a.batch, split = id / a.batch;
  const int len = min(max(a.len[b], 0), a.width << c.shift);
  const int t0 = a.cu ? a.cu[b] : b * a.max_q;
  const int m = a.cu ? min(max(a.cu[b + 1] - t0, 0), a.max_q) : a.max_q;
  const int rows = m * a.group, row_begin = row_tile * kManyRows;
  const int begin = split * kStep, stride = a.splits * kStep, first_q = a.len[b] - m;
  if (row_begin >= rows || t0 < 0 || t0 > a.total_q - m || (begin >= len && split > 0)) return;
  const int prefix = a.prefix ? min(max(a.prefix[b], 0), len) : 0;
  auto limit_of = [&](int row) { return max(min(first_q + row / a.group + 1, len), prefix); };
  const int end = limit_of(min(row_begin + kManyRows, rows) - 1);
  const int steps = end > begin ? (end - begin + stride - 1) / stride : 0;

  const int wave_row = row_begin + wave * 32;
  const bool idle = wave_row >= rows;            // nothing to attend, but its share of the tokens to unpack
  const int least = limit_of(min(wave_row, rows - 1));
  RowState st;
  typename Q::frag q[8][1];
  const int row = wave_row + x;
  const bool on = row < rows;
  {
    const int i = row / a.group, hq = head * a.group + row % a.group;
    st.limit = on ? limit_of(row) : 0;
    st.m = -INFINITY;
    st.l = 0.f;
    st.slope = kMode == kBiased && a.slopes && on ? a.slopes[hq] * kLog2e : 0.f;
    st.q_at = kMode == kBiased && on ? (a.q_pos ? a.q_pos[t0 + i] : first_q + i) : 0;
    load_query<DT, 8>(q, a.Q + (size_t)(t0 + i) * a.qst + (size_t)hq * a.qsh, on, [g](int k) { return 16 * k + 8 * g; });
  }
  const float factor = kMode == kPlain ? a.scale * kLog2e : a.scale;
  // E4M3's scales are powers of two and go into V's bf16 operands for nothing (of a scale that is none, from a pool that was
  // filled elsewhere, what is left over goes into the weights).  Integers are the codes, and the weights are multiplied.
  constexpr bool kTrueV = FMT == SPINDLE_E4M3;

  f16v o[4], s[2];                                // [32 dimensions][..], [32 tokens][..]; the row is lane % 32
  frag p[4][N::kP];                              // weights of 16 tokens
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
#pragma unroll
    for (int part = 0; part < N::kP; ++part) p[i][part] = __builtin_bit_cast(frag, u4{0, 0, 0, 0});
  }

  // ---- what this thread brings of each half of a step: a piece of 16 bytes of one token of K, 4 dimensions of 4 tokens of V
  const int32_t *table = a.table + (size_t)b * a.width;
  const int kx = tid & 15, kc = (tid >> 4) & 7, ks0 = tid >> 7;           // token in its 16, piece (a step of K's), which 16
  const int vd = tid & 31, vg = tid >> 5;                                 // tokens 4 vg + 0..3, dimensions 4 vd + 0..3
  char *const k_to = lds + (kc * 64 + 16 * ks0 + kx) * 16;
  // V's operand of 16 tokens: lane group g has tokens 4 g + 0..3 and 8 + 4 g + 0..3, as the logits leave the weights.  Lanes
  // are exchanged by tile, or the threads that write side by side would meet in the same banks.
  char *const v_to = lds + 2 * kBuffer + (((vg >> 2) * 4 + (vd >> 3)) * 64 + (vg & 1) * 32) * 16 + ((vg >> 1) & 1) * 8;
  const int v_lane0 = 4 * (vd & 7), v_turn = vd >> 3;
  const uint32_t k_lane = (16 * ks0 + kx) * kHeadDim + 16 * kc, v_lane = 4 * vg * kHeadDim + 4 * vd;
  u4 raw_k[2];
  uint32_t raw_v[2][4];
  struct Place {
    bool there;
    uint32_t number;
    float ks, vs;
  } now[2], next[2];
  // (behind the end the last page, which is then not used: a lookup is no branch)
  const int last = max(end, 1) - 1;
  int page[2];
  auto look_up = [&](int t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) page[h] = uniform_load_at(table, (uint32_t)min(t + 32 * h, last) >> c.shift);
  };
  // (for an absent page the loads go to page 0, and what they bring is not used)
  auto fetch = [&](int t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      next[h].there = t + 32 * h < end && (uint32_t)page[h] < (uint32_t)c.n_pages;
      const uint32_t number = page_number(c, next[h].there ? page[h] : 0, head);
      const uint64_t at = page_bytes(c, number, (t + 32 * h) & (c.P - 1));
      const uint8_t *const kp = c.k + at, *const vp = c.v + at;
      next[h].number = number;
      next[h].ks = uniform_load_at(c.ks, number);
      next[h].vs = uniform_load_at(c.vs, number);
      raw_k[h] = *reinterpret_cast<const u4 *>(kp + k_lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) raw_v[h][j] = *reinterpret_cast<const uint32_t *>(vp + (v_lane + j * kHeadDim));
    }
  };
  auto unpack = [&](int t, int buffer) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      asm volatile("" : "+v"(raw_k[h]));
      char *const to = k_to + buffer * kBuffer + h * (8 * kFrag);
      *reinterpret_cast<typename Q::frag *>(to) = Q::template codes<FMT>(raw_k[h][0], raw_k[h][1]);
      *reinterpret_cast<typename Q::frag *>(to + 512) = Q::template codes<FMT>(raw_k[h][2], raw_k[h][3]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(raw_v[h][j]));
      const int here = next[h].there ? len - t - 32 * h - 4 * vg : 0;  // what lies behind the last token may be anything
#pragma unroll
      for (int j = 0; j < 4; ++j) raw_v[h][j] = j < here ? raw_v[h][j] : 0;
      uint32_t col[4];
      transpose4(raw_v[h][0], raw_v[h][1], raw_v[h][2], raw_v[h][3], col);
      char *const to = v_to + buffer * kBuffer + h * (8 * kFrag);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {           // (8 bytes of each of two dimensions at a time)
        const u4 w = __builtin_bit_cast(u4, Weights::codes<FMT>(col[e], col[e + 1], kTrueV && next[h].there ? operand_scale(next[h].vs) : 1.f));
        *reinterpret_cast<u2 *>(to + ((v_lane0 + e) ^ v_turn) * 16) = u2{w[0], w[1]};
        *reinterpret_cast<u2 *>(to + ((v_lane0 + e + 1) ^ v_turn) * 16) = u2{w[2], w[3]};
      }
    }
  };

  look_up(begin);
  fetch(begin);
  look_up(begin + stride);
  unpack(begin, 0);
  now[0] = next[0], now[1] = next[1];
  fetch(begin + stride);
  look_up(begin + 2 * stride);
  const char *const from_k = lds + lane * 16;
  int v_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v_off[i] = 2 * kBuffer + (g * 32 + (x ^ i)) * 16;
  auto times_v = [&](int n) {                    // O += V(n) P
    const char *const from = lds + (n & 1) * kBuffer;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      frag vv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) vv[i] = *reinterpret_cast<const frag *>(from + v_off[i] + (u * 4 + i) * kFrag);
#pragma unroll
      for (int part = N::kP - 1; part >= 0; --part)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = Weights::mma32(vv[i], p[u][part], o[i]);
    }
  };
  __syncthreads();
  if (idle) {
    for (int n = 0; n < steps; ++n) {
      unpack(begin + (n + 1) * stride, (n + 1) & 1);
      fetch(begin + (n + 2) * stride);
      look_up(begin + (n + 3) * stride);
      __syncthreads();
    }
    return;
  }
  for (int n = 0; n < steps; ++n) {
    const int t = begin + n * stride;
    {
      const char *const from = from_k + (n & 1) * kBuffer;
      const f16v zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) s[h] = Q::mma32(*reinterpret_cast<const typename Q::frag *>(from + (h * 8 + k) * kFrag), q[k][0], k ? s[h] : zero);
    }
    unpack(t + stride, (n + 1) & 1);
    const Place here[2] = {now[0], now[1]};
    now[0] = next[0], now[1] = next[1];
    fetch(t + 2 * stride);
    look_up(t + 3 * stride);
    {
      // (what is no logit in the end must not be a NaN before)
      const bool there[2] = {here[0].there, here[1].there};
      const float kf[2] = {there[0] ? fmaxf(factor * here[0].ks, kTinyScale) : 1.f, there[1] ? fmaxf(factor * here[1].ks, kTinyScale) : 1.f};
      const float slope[2] = {logit_slope<kMode>(kf[0], a), logit_slope<kMode>(kf[1], a)}, offset = logit_offset<kMode>(a);
      // an integer's V scale goes into the exponent, and out of the sum again; what is far from 1 is multiplied in at the end,
      // where neither the exponent's bits nor the sum can suffer
      float log_v[2] = {0.f, 0.f}, per_v[2] = {1.f, 1.f}, rest_v[2] = {1.f, 1.f};
      const bool odd_v = kTrueV && (operand_scale(here[0].vs) != here[0].vs || operand_scale(here[1].vs) != here[1].vs);
      bool far_v = false;
      if (!kTrueV) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float v = there[h] ? here[h].vs : 1.f, log = __builtin_amdgcn_logf(v);
          if (__builtin_fabsf(log) <= 24.f) {
            log_v[h] = log;
            per_v[h] = __builtin_amdgcn_exp2f(-log);
          } else {
            rest_v[h] = v;
            far_v = true;
          }
        }
      }
      // token of logit e of half h: t + 32 h + 8 (e / 4) + 4 g + e % 4
      if (kMode != kPlain) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int32_t *pos = kMode == kBiased && c.pos ? c.pos + (((uint64_t)here[h].number << c.shift) + (uint32_t)((t + 32 * h) & (c.P - 1))) : nullptr;
          if (pos) {
            int k_at[16];
#pragma unroll
            for (int e = 0; e < 16; e += 4) load_positions(pos + 2 * e + 4 * g, k_at + e);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = raw_logit<kMode>(s[h][e], kf[h], a, st, k_at[e]);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = raw_logit<kMode>(s[h][e], kf[h], a, st, t + 32 * h + 8 * (e >> 2) + 4 * g + (e & 3));
          }
        }
      }
      if (t + kStep > least || !there[0] || !there[1] || odd_v) {   // (one branch for all that is rare)
        if (odd_v) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!there[h] || !(here[h].vs > 0.f)) continue;
            log_v[h] = __builtin_amdgcn_logf(here[h].vs * (1.f / operand_scale(here[h].vs)));   // 0 of a power of two
            per_v[h] = __builtin_amdgcn_exp2f(-log_v[h]);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (t + 32 * h + 8 * (e >> 2) + 4 * g + (e & 3) >= st.limit || !there[h]) s[h][e] = -INFINITY;
      }
      float top[2] = {s[0][0], s[1][0]};
#pragma unroll
      for (int e = 1; e < 16; ++e) top[0] = larger(top[0], s[0][e]), top[1] = larger(top[1], s[1][e]);
      bool scaled;
      const float back = gather(st, over_halves_max(larger(__builtin_fmaf(top[0], slope[0], offset), __builtin_fmaf(top[1], slope[1], offset))), &scaled);
      const float base = offset - (st.m == -INFINITY ? 0.f : st.m + kSlack);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float from = base + log_v[u >> 1];
        float w[8], sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][8 * (u & 1) + j], slope[u >> 1], from));
          sum += w[j];
        }
        st.l = __builtin_fmaf(sum, per_v[u >> 1], st.l);
        if (!kTrueV && far_v) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] *= rest_v[u >> 1];
        }
        Weights::split<N::kP>(w, p[u]);
      }
      if (scaled) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= back;
      }
      times_v(n);
    }
    __syncthreads();
  }

  // dimension 32 i + 8 k + 4 g + e of row x is o[i][4 k + e]
  const float l = over_halves_sum(st.l);
  if (!on) return;
  const float inv = l > 0.f ? 1.f / l : l;                          // a row that saw nothing: 0; NaN stays
  const size_t out_row = (size_t)(t0 + row / a.group) * a.heads_q + head * a.group + row % a.group;
  if (a.splits == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        T e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = Elem<DT>::from_float(o[i][4 * k + j] * inv);
        __builtin_memcpy(__builtin_assume_aligned(a.out + (out_row * kHeadDim + 32 * i + 8 * k + 4 * g) * sizeof(T), 8), e, sizeof(e));
      }
    if (a.lse && g == 0) a.lse[out_row] = lse_of(st.m, l);
  } else {
    float *po = a.part_o + (out_row * a.splits + split) * kHeadDim + 4 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<f4 *>(po + 32 * i + 8 * k) = f4{o[i][4 * k] * inv, o[i][4 * k + 1] * inv, o[i][4 * k + 2] * inv, o[i][4 * k + 3] * inv};
    if (g == 0) a.part_ml[out_row * a.splits + split] = float2{st.m, l};
  }
}

template <int DT, int FMT>
spindle_status launch(const AttendArgs &a, int mode, unsigned blocks, hipStream_t st) {
  constexpr int bytes = 4 * kBuffer;             // the 64 KB that need no raised limit
  if (mode == kPlain) hipLaunchKernelGGL((attend_rows<DT, FMT, kPlain>), dim3(blocks), dim3(kThreads), bytes, st, a);
  else if (mode == kCapped) hipLaunchKernelGGL((attend_rows<DT, FMT, kCapped>), dim3(blocks), dim3(kThreads), bytes, st, a);
  else hipLaunchKernelGGL((attend_rows<DT, FMT, kBiased>), dim3(blocks), dim3(kThreads), bytes, st, a);
  return SPINDLE_OK;
}

}  // namespace

spindle_status launch_attend_rows(const AttendArgs &a, int dtype, int format, int mode, unsigned blocks, hipStream_t st) {
  if (dtype == SPINDLE_F16)
    return format == SPINDLE_E4M3 ? launch<SPINDLE_F16, SPINDLE_E4M3>(a, mode, blocks, st) : launch<SPINDLE_F16, SPINDLE_I8>(a, mode, blocks, st);
  return format == SPINDLE_E4M3 ? launch<SPINDLE_BF16, SPINDLE_E4M3>(a, mode, blocks, st) : launch<SPINDLE_BF16, SPINDLE_I8>(a, mode, blocks, st);
}

}  // namespace spindle
