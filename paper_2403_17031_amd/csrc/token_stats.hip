// Log-probabilities of given tokens, entropies and most likely alternatives of rows of hidden states under an output matrix,
// and the gradient of the first two: logits l = h W^T (fp32 sums), z = l / temperature,
//   lse = log sum_v exp z_v,  logprob = z_y - lse,  entropy = log S0 - S1 / S0
//   with S0 = sum exp(z - max), S1 = sum exp(z - max) (z - max),
//   dz_v = (g ([v = y] - p_v) - e p_v (log p_v + entropy)) / temperature,  dh = dz W,  dW = dz^T h.
//
// Forward: the product's epilogue leaves (max, S0, S1) of every part (the 64 columns of a wave) of a row, so without alternatives
// no logit is stored.  With them: an entry among a row's k largest lies in one of the k parts whose maxima are largest (ties:
// the lower part, as the lower id among equals), since each part before its own in that order holds an entry before it.  So the
// first column tiles store their logits, which bounds the k-th largest maximum of each row, and the others store the
// parts that reach the bound, 16,384 rows at a time (few rows: all is stored).  The last kernel merges the parts' sums, picks
// those parts, then the k entries among their 64 k logits.
//
// Backward: the first product's epilogue forms dz, rounded to the operands' type: products of 16-bit operands are what the
// matrix cores run at full rate (float is a tenth), and the rounding, half a step of 2^-8 or 2^-11 relative, is that of the results
// in the same type.  Both roundings together: d_hidden is off by 0.23 % (bfloat16, 13,568 rows of a 2.8B model's width; 0.17 % if it
// were only rounded at the end).  dh and dW read dz row-major and K-major, W and h as they lie.
//
// What bounds it: few rows read W (1 row, 50,304 x 2,560 in bfloat16: 62 us, 4.2 TB/s with the finishing kernel and the launches; a copy
// reaches 5.0); many are matrix products (13,568 rows: 2.74 ms without alternatives, 1,275 TFLOP/s of the 1,290 that a
// library product of this size reaches here; the gradient 8.75 ms, 1,200).
#include <algorithm>
#include <cmath>

#include "common.h"
#include "product_tile.h"
#include "token_stats.h"

namespace rlhf {

namespace {

constexpr int kPart = 64;  // columns of a part

__device__ __forceinline__ uint32_t order_key(float v) {  // larger for larger values, -0 as +0, NaN below all
  const uint32_t b = __float_as_uint(v + 0.0f);
  return v != v ? 0u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

struct StatsArgs {
  const void *h, *w;
  uint32_t ldh, ldw;
  int T, V, d;
  const int32_t* targets;
  float inv_t;
  float *pmax, *ps0, *ps1;  // [part][T]
  float* ztgt;              // [T], the target's logit
  float* logits;            // [T][ldl] or null
  int ldl, tile0, tiles_n;  // column tiles of this launch
  const float* thr;         // [T] or null: only parts whose maximum is not below their row's are stored
};

// A tile of logits in the accumulators and what is kept of it.  The epilogue is vector work (a maximum, an exponential and seven more
// instructions an entry) that the matrix cores wait for: 9 us of a tile of 256 x 256, whose product takes 1.7 us a stage, which is
// why K = 768 runs at two thirds of the rate that K = 2,560 does.  13,568 x 50,304, K = 2,560: 2.6 ms of the call's 2.74.
template <typename T, typename S>
__global__ void __launch_bounds__(64 * S::waves, pt_waves_eu<S>) stats_kernel(StatsArgs a) {
  PT_STAGES(S)
  constexpr int MT = S::MT;
  const int nb_m = (a.T + S::rows - 1) / S::rows;
  const int item = pt_item(nb_m * a.tiles_n);
  if (item < 0) return;
  int tm, tn;
  pt_tile_pos(item, nb_m, a.tiles_n, tm, tn);
  tn += a.tile0;
  pt_f32x16 acc[2][MT];
  PT_PRODUCT(T, false, false, a.h, a.ldh, tm * S::rows, a.T, a.w, a.ldw, tn * S::cols, a.V, 0, a.d, nullptr);
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hf = lane >> 5;
  if (pt_done<S>(wave)) return;
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
  if (col0 >= a.V) return;
  const int part = col0 / kPart;
  const float c2 = a.inv_t * 1.44269504088896341f;
  // the sums of a part; `all`: its 64 columns exist (without it, 32 masks would be held in registers)
  auto sums = [&](auto all) {
    constexpr bool ALL = decltype(all)::value;
    int lim = a.V - col0;
    asm volatile("" : "+s"(lim));
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int row = row0 + 32 * i + l32;
      const bool in = row < a.T;
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, ALL || pt_col(j, e, hf) < lim ? acc[j][i][e] : -INFINITY);
      m = half_max(m);
      // s0: the sum, less: what of it is below 1 each, so without the largest entries, whose count is the difference
      float s0 = 0.f, less = 0.f, s1 = 0.f;
      if (m > -INFINITY) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float t = (acc[j][i][e] - m) * c2;
            float x = __builtin_amdgcn_exp2f(t);  // (of NaN, which the maximum passes over, NaN)
            if (!ALL) x = pt_col(j, e, hf) < lim ? x : 0.f;
            s0 += x;
            less += __builtin_amdgcn_fractf(x);
            s1 = fmaf(x, fmaxf(t, -1e30f), s1);  // (0 times -infinity)
          }
      } else {  // -infinity alone, or NaN
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (pt_col(j, e, hf) < lim && acc[j][i][e] != acc[j][i][e]) s0 = acc[j][i][e];
      }
      s0 = half_sum(s0);
      less = half_sum(less);
      s1 = half_sum(s1);
      if (in && hf == 0) {
        const size_t at = (size_t)part * a.T + row;
        a.pmax[at] = m;
        a.ps0[at] = (rintf(s0 - less) - 1.f) + less;
        a.ps1[at] = s1 * 0.69314718055994531f;
      }
      if (a.thr) {  // few rows keep their part: straight from the accumulators
        const bool keep = in && !(m < a.thr[min(row, a.T - 1)]);
        if (__ballot(keep)) {
          float* const o = a.logits + (size_t)row * a.ldl + col0 + 4 * hf;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (keep)
                *(pt_f32x4*)(o + 32 * j + 8 * q) =
                    pt_f32x4{acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
        }
      }
      // the target's logit, where one of the wave's rows has it here
      const int tcol = in ? a.targets[row] - col0 : -1;  // (an absent target is negative)
      if (__ballot((unsigned)tcol < 64u)) {
        float zt = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) zt = pt_col(j, e, hf) == tcol ? acc[j][i][e] : zt;
        if ((unsigned)tcol < 64u && ((tcol >> 2) & 1) == hf) a.ztgt[row] = zt;
      }
    }
  };
  if (a.V - col0 >= 64) sums(std::true_type{});
  else sums(std::false_type{});
  if (a.logits && !a.thr) {  // (columns up to the row stride, a multiple of 64, exist)
    pt_hand_out<4, MT>(PT_WAVE_LDS, lane, acc, PtNothing(), [&](int r, int c, pt_f32x4 v, int) {
      if (row0 + r < a.T) *(pt_f32x4*)(a.logits + (size_t)(row0 + r) * a.ldl + col0 + c) = v;
    });
  }
}

// (max, S0 - 1, S1) of a set of entries (none: S0 = 0).  S0 is kept less the largest entry's 1, so that a token which has nearly
// everything gets its log-probability, -log S0, to the bits of what the others have.
struct Stat {
  float m, over, s1;
};
__device__ __forceinline__ Stat stat_merge(Stat a, Stat b, float inv_t) {
  if (b.m > a.m) {
    const Stat x = a;
    a = b;
    b = x;
  }
  const float s0 = 1.f + b.over;
  if (b.m == -INFINITY) {  // nothing, or NaN alone
    a.over += s0;
    return a;
  }
  const float t = (b.m - a.m) * inv_t, f = __expf(t);
  a.over = fmaf(f, s0, a.over);
  if (f != 0.f) a.s1 = fmaf(f, fmaf(s0, t, b.s1), a.s1);
  return a;
}

// 4-byte words of LDS of a wave that looks for alternatives
__host__ __device__ constexpr int finish_words(int top) { return top * (kPart + 2) < 160 ? 160 : top * (kPart + 2); }

struct FinishArgs {
  const float *pmax, *ps0, *ps1, *ztgt, *logits;
  const int32_t* targets;
  int T, V, parts, ldl, top;
  float inv_t, inv_lo;  // (inv_lo: what inv_t was rounded by)
  float *logprob, *entropy, *lse;
  int32_t* top_ids;
  float* top_logprob;
};

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  auto step = [&](auto o) { v = max(v, (uint32_t)lane_xor<decltype(o)::value>((int)v)); };
  step(std::integral_constant<int, 32>{});
  step(std::integral_constant<int, 16>{});
  step(std::integral_constant<int, 8>{});
  step(std::integral_constant<int, 4>{});
  step(std::integral_constant<int, 2>{});
  step(std::integral_constant<int, 1>{});
  return v;
}

// The k first of n keys in LDS in the order (key descending, place ascending), one by one: lane l has the places l, l + 64, ...; every
// lane keeps the first of its own that is left, and the lane whose key is taken looks for its next (eight loads at a time
// under way: a loop that waits for each is most of the kernel).  take(rank, key, place) is called by all lanes.
template <typename F>
__device__ __forceinline__ void wave_select(const uint32_t* keys, int n, int k, int lane, F take) {
  uint32_t bk = 0, bi = ~0u;
  auto look = [&](uint32_t lk, uint32_t li) {  // this lane's first behind (lk, li)
    bk = 0;
    bi = ~0u;
    for (int i0 = lane; i0 < n; i0 += 512) {
      uint32_t x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = keys[min(i0 + 64 * u, n - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint32_t i = i0 + 64 * u;
        const bool behind = i < (uint32_t)n && (x[u] < lk || (x[u] == lk && i > li));
        if (behind && (x[u] > bk || bi == ~0u)) bk = x[u], bi = i;
      }
    }
  };
  look(~0u, 0);  // (no key is ~0: that would be a NaN)
  for (int r = 0; r < k; ++r) {
    const uint32_t top = wave_max_u32(bk);
    const uint32_t first = ~wave_max_u32(bk == top ? ~bi : 0u);
    take(r, top, first);
    if (bi == first) look(top, first);
  }
}

// A value that at least k of the lanes' items are not below, and few more: the k-th largest of the lanes' largest (k <= 64).
__device__ __forceinline__ uint32_t wave_bound(uint32_t largest, int k) {
  int above = 0;
#pragma unroll
  for (int l = 0; l < 64; ++l) above += (uint32_t)__builtin_amdgcn_readlane((int)largest, l) > largest ? 1 : 0;
  return ~wave_max_u32(above < k ? ~largest : 0u);
}
__device__ __forceinline__ int lanes_below(uint64_t mask) {  // set bits below this lane's
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

constexpr int kQuickTop = 32, kQuickParts = 32;

// The alternatives of one row by a wave, quickly: the parts whose maximum reaches a bound that k part maxima reach; of their
// logits those that reach a bound that k of them reach; and the ranks of these, at most 64, by comparing all with all.
// False, with nothing written, where ties or an odd spread leave more than fit.
template <int NB>
__device__ __forceinline__ bool rank_logits(const float* logits, int V, const int* sel, int parts, int top, int lane, uint32_t* keep_key,
                                            int* keep_col, float inv_t, float m, float ls, int32_t* ids, float* lps) {
  uint32_t x[NB], largest = 0;
  int col[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    col[j] = sel[min(j, parts - 1)] * kPart + lane;
    x[j] = __float_as_uint(logits[min(col[j], V - 1)]);
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const bool in = j < parts && col[j] < V;
    x[j] = in ? order_key(__uint_as_float(x[j])) : 0u;
    if (!in) col[j] = -1;
    largest = max(largest, x[j]);
  }
  const uint32_t bound = wave_bound(largest, top);
  int n = 0;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const bool keep = col[j] >= 0 && x[j] >= bound;
    const uint64_t who = __ballot(keep);
    const int at = n + lanes_below(who);
    if (keep && at < 64) {
      keep_key[at] = x[j];
      keep_col[at] = col[j];
    }
    n += __popcll(who);
  }
  if (n > 64) return false;
  PT_WAVE_LDS_FENCE();
  const uint32_t key = keep_key[min(lane, n - 1)];
  const int c = keep_col[min(lane, n - 1)];
  int rank = 0;
  for (int l = 0; l < n; ++l) {
    const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key, l);
    rank += k > key || (k == key && __builtin_amdgcn_readlane(c, l) < c) ? 1 : 0;
  }
  if (lane < n && rank < top) {
    ids[rank] = c;
    lps[rank] = (order_value(key) - m) * inv_t - ls;
  }
  return true;
}

// The places (ascending, up to `most`) of the keys that reach the bound of k of them; returns how many reach it.
__device__ __forceinline__ int bounded_places(const uint32_t* keys, int n, int k, int most, int lane, int* places) {
  uint32_t largest = 0;
  for (int i0 = lane; i0 < n; i0 += 512)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint32_t x = keys[min(i0 + 64 * u, n - 1)];
      largest = max(largest, i0 + 64 * u < n ? x : 0u);
    }
  const uint32_t bound = wave_bound(largest, k);
  int found = 0;
  for (int i0 = 0; i0 < n; i0 += 512) {
    uint32_t x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = keys[min(i0 + 64 * u + lane, n - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + 64 * u + lane;
      const bool keep = i < n && x[u] >= bound;
      const uint64_t who = __ballot(keep);
      const int at = found + lanes_below(who);
      if (keep && at < most) places[at] = i;
      found += __popcll(who);
    }
  }
  return found;
}

// Block: R rows, 256 / R threads to each for the sums; then a wave per row for the alternatives.  Bound by the latency of its few
// dependent reads: 13,568 rows of 786 parts with eight alternatives 86 us (the parts' 128 MB would take 26; 120 where neighbours, whose rows
// share lines, run on different XCDs), 1,003 rows 14, one row 9.
// LDS: the keys of the rows' part maxima [R][parts | 1] (with alternatives), then of each wave its candidates' [top * 64] and the
// parts [top], as chosen and by id, or (the quick way) the parts [32] and the keys and ids of what is ranked [64].
template <int R>
__global__ void __launch_bounds__(256) stats_finish_kernel(FinishArgs a) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  __shared__ float sh[3][4][16];
  __shared__ float row_max[16], row_log[16];
  constexpr int G = 256 / R;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = tid % R, g = tid / R, P = a.parts | 1;
  const int block = pt_item((a.T + R - 1) / R);  // (neighbours on one XCD: their rows share the lines of the parts' sums)
  if (block < 0) return;
  const int row = block * R + r;
  const bool in = row < a.T;
  uint32_t* const pm = (uint32_t*)dyn;
  Stat s = {-INFINITY, -1.f, 0.f};
  if (in) {
    for (int p = g; p < a.parts; p += G) {
      const size_t at = (size_t)p * a.T + row;
      const Stat x = {a.pmax[at], a.ps0[at], a.ps1[at]};
      if (a.top) pm[r * P + p] = order_key(x.m);
      s = stat_merge(s, x, a.inv_t);
    }
  }
  // over the row's threads: the maximum, then the sums brought to it, in a fixed order
  auto over = [&](float v, auto op, int k) {
    if (R <= 1) v = op(v, lane_xor<1>(v));
    if (R <= 2) v = op(v, lane_xor<2>(v));
    if (R <= 4) v = op(v, lane_xor<4>(v));
    if (R <= 8) v = op(v, lane_xor<8>(v));
    v = op(v, lane_xor<16>(v));
    v = op(v, lane_xor<32>(v));
    if (lane < R) sh[k][wave][lane] = v;
    __syncthreads();
    return op(op(sh[k][0][r], sh[k][1][r]), op(sh[k][2][r], sh[k][3][r]));
  };
  const float m = over(s.m, [](float x, float y) { return fmaxf(x, y); }, 0);
  // the largest entry's 1 is left out once, with the first thread of the row whose own maximum it is
  auto holder = [&] {
    int first = s.m == m ? g : 256;
    if (R <= 1) first = min(first, lane_xor<1>(first));
    if (R <= 2) first = min(first, lane_xor<2>(first));
    if (R <= 4) first = min(first, lane_xor<4>(first));
    if (R <= 8) first = min(first, lane_xor<8>(first));
    first = min(first, lane_xor<16>(first));
    first = min(first, lane_xor<32>(first));
    if (lane < R) sh[1][wave][lane] = (float)first;
    __syncthreads();
    return (int)fminf(fminf(sh[1][0][r], sh[1][1][r]), fminf(sh[1][2][r], sh[1][3][r])) == g;
  };
  const bool holds = holder();
  Stat mine = s;
  if (!holds) mine = stat_merge(Stat{m, 0.f, 0.f}, s, a.inv_t);  // (over: without the 1 that it then has too much)
  __syncthreads();
  const auto add = [](float x, float y) { return x + y; };
  const float excess = over(mine.over, add, 1), s1 = over(mine.s1, add, 2);
  if (g == 0 && in) {
    const float ls = log1pf(excess);
    row_max[r] = m;
    row_log[r] = ls;
    a.lse[row] = fmaf(m, a.inv_t, fmaf(fmaxf(m, -1e30f), a.inv_lo, ls));
    a.entropy[row] = ls - s1 / (1.f + excess);
    const int y = a.targets[row];
    a.logprob[row] = y >= 0 && y < a.V ? (a.ztgt[row] - m) * a.inv_t - ls : 0.f;
  }
  if (!a.top) return;
  __syncthreads();
  const int kp = min(a.top, a.parts);
  uint32_t* const cand = pm + R * P + wave * finish_words(a.top);
  int *const chosen = (int*)(cand + a.top * kPart), *const sel = chosen + a.top;
  for (int q = wave; q < R; q += 4) {
    const int t = block * R + q;
    if (t >= a.T) break;
    if (a.top <= kQuickTop) {
      int *const places = (int*)cand, *const cols = places + kQuickParts + 64;
      uint32_t* const keys = cand + kQuickParts;
      const int n = bounded_places(pm + q * P, a.parts, kp, kQuickParts, lane, places);
      PT_WAVE_LDS_FENCE();
      const float* const row_logits = a.logits + (size_t)t * a.ldl;
      int32_t* const ids = a.top_ids + (size_t)t * a.top;
      float* const lps = a.top_logprob + (size_t)t * a.top;
      bool done = false;
      if (n <= 12) done = rank_logits<12>(row_logits, a.V, places, n, a.top, lane, keys, cols, a.inv_t, row_max[q], row_log[q], ids, lps);
      else if (n <= kQuickParts) done = rank_logits<kQuickParts>(row_logits, a.V, places, n, a.top, lane, keys, cols, a.inv_t, row_max[q], row_log[q], ids, lps);
      PT_WAVE_LDS_FENCE();
      if (done) continue;
    }
    wave_select(pm + q * P, a.parts, kp, lane, [&](int k, uint32_t, uint32_t i) {
      if (lane == 0) chosen[k] = (int)i;
    });
    PT_WAVE_LDS_FENCE();
    if (lane < kp) {  // in the order of their ids, so that a candidate's place orders as its id does
      const int mine = chosen[lane];
      int rank = 0;
      for (int k = 0; k < kp; ++k) rank += chosen[k] < mine;
      sel[rank] = mine;
    }
    PT_WAVE_LDS_FENCE();
    for (int k = 0; k < kp; ++k) {  // (ids past the vocabulary come last and are not reached)
      const int col = sel[k] * kPart + lane;
      cand[k * kPart + lane] = col < a.V ? order_key(a.logits[(size_t)t * a.ldl + col]) : 0u;
    }
    PT_WAVE_LDS_FENCE();
    const float m = row_max[q], ls = row_log[q];
    wave_select(cand, kp * kPart, a.top, lane, [&](int k, uint32_t key, uint32_t i) {
      if (lane == 0) {
        a.top_ids[(size_t)t * a.top + k] = sel[i >> 6] * kPart + (int)(i & 63);
        a.top_logprob[(size_t)t * a.top + k] = (order_value(key) - m) * a.inv_t - ls;
      }
    });
    PT_WAVE_LDS_FENCE();
  }
}

// thr[row] = a bound that `top` of the row's first `parts` maxima reach: no part below it can hold one of the row's top entries.
// (13,568 rows, 112 parts: 15 us.)
__global__ void __launch_bounds__(256) stats_threshold_kernel(const float* __restrict__ pmax, int T, int parts, int top, float* __restrict__ thr) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = parts | 1;
  uint32_t* const pm = (uint32_t*)dyn;
  const int block = pt_item((T + 15) / 16);
  if (block < 0) return;
  for (int i = tid; i < 16 * parts; i += 256) {
    const int row = block * 16 + (i & 15);
    if (row < T) pm[(i & 15) * P + (i >> 4)] = order_key(pmax[(size_t)(i >> 4) * T + row]);
  }
  __syncthreads();
  for (int q = wave; q < 16; q += 4) {
    const int row = block * 16 + q;
    if (row >= T) break;
    uint32_t largest = 0;
    for (int i = lane; i < parts; i += 64) largest = max(largest, pm[q * P + i]);
    const uint32_t bound = wave_bound(largest, top);
    if (lane == 0) thr[row] = bound ? order_value(bound) : -INFINITY;
  }
}

// dst [rows_to][ldd] = src [rows][cols] (row stride lds), zero beyond either; 16 bytes of dst a thread.  Rows of src may start at
// any element: its loads need no more alignment than that.  (50,277 x 1,037 halves: 37 us, 5.8 TB/s, some of it from the last cache.)
template <typename T>
__global__ void __launch_bounds__(256)
    pack_rows_kernel(const T* __restrict__ src, size_t lds, int rows, int cols, T* __restrict__ dst, int ldd, int rows_to) {
  constexpr int E = 16 / (int)sizeof(T);
  typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t loose;
  const int per_row = ldd / E;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
  const int c = (int)(i - row * per_row) * E;
  if (row >= (size_t)rows_to) return;
  const T* const s = src + row * lds + c;
  T v[E];
  if (row < (size_t)rows && c + E <= cols) {
    const loose x = *(const loose*)s;
    __builtin_memcpy(v, &x, 16);
  } else {
#pragma unroll
    for (int u = 0; u < E; ++u) v[u] = row < (size_t)rows && c + u < cols ? s[u] : (T)0.f;
  }
  __builtin_memcpy(__builtin_assume_aligned(dst + row * ldd + c, 16), v, 16);
}

// scale[0] = the power of two that brings the largest |dz| a row could have (|g| + 14 |e|, |log p + H| p being less) to 2^11 .. 2^12, well
// inside fp16's range at either end; scale[1] = its reciprocal.
__global__ void __launch_bounds__(1024) grad_scale_kernel(const int32_t* __restrict__ targets, const float* __restrict__ g,
                                                          const float* __restrict__ e, int T, int V, float inv_t, float* __restrict__ scale) {
  __shared__ float sh[16];
  float m = 0.f;
  for (int t = threadIdx.x; t < T; t += 1024) {
    const float x = (targets[t] >= 0 && targets[t] < V ? fabsf(g[t]) : 0.f) + (e ? 14.f * fabsf(e[t]) : 0.f);
    if (x < INFINITY) m = fmaxf(m, x);
  }
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) m = fmaxf(m, sh[i]);
    m *= inv_t;
    int x = 12;
    if (m > 0.f && m < INFINITY) (void)frexpf(m, &x);  // m < 2^x
    x = min(max(12 - x, -60), 60);
    scale[0] = ldexpf(1.f, x);
    scale[1] = ldexpf(1.f, -x);
  }
}

struct DzArgs {
  const void *h, *w;
  uint32_t ldh, ldw;
  int T, V, d;
  const int32_t* targets;
  const float *lse, *entropy, *g, *e;  // e may be null
  const float* scale;                  // null: 1
  float inv_t, inv_lo;   // (see FinishArgs)
  void* dz;  // [rows][ldz], zero from T and V on
  int ldz, rows, tile0, tiles_n;
};

// A tile of logits once more, and dz in place of it.  13,568 x 50,304, K = 2,560, bfloat16: 3.1 ms, 1,125 TFLOP/s: the product's 2.7 and the
// epilogue, 1.4 GB of dz included, of which a CU that has one large tile overlaps nothing with its next.
template <typename T, typename S>
__global__ void __launch_bounds__(64 * S::waves, pt_waves_eu<S>) dz_kernel(DzArgs a) {
  PT_STAGES(S)
  constexpr int MT = S::MT;
  const int nb_m = (a.T + S::rows - 1) / S::rows;
  const int item = pt_item(nb_m * a.tiles_n);
  if (item < 0) return;
  int tm, tn;
  pt_tile_pos(item, nb_m, a.tiles_n, tm, tn);
  tn += a.tile0;
  pt_f32x16 acc[2][MT];
  PT_PRODUCT(T, false, false, a.h, a.ldh, tm * S::rows, a.T, a.w, a.ldw, tn * S::cols, a.V, 0, a.d, nullptr);
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hf = lane >> 5;
  if (pt_done<S>(wave)) return;
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
  if (row0 >= a.rows || col0 >= a.ldz) return;
  const float s = (a.scale ? a.scale[0] : 1.f) * a.inv_t;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = min(row0 + 32 * i + l32, a.T - 1);
    const int t = a.targets[row], y = t < a.V ? t : -1;
    const float g = y >= 0 ? a.g[row] * s : 0.f, e = a.e ? a.e[row] * s : 0.f;
    const float lse = a.lse[row], H = a.entropy[row];  // (H: anything without e)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        // (a finite log p: 0 times infinity; the reciprocal's rounding is one sign over a row, which float would show)
        const float logp = fmaf(acc[j][i][x], a.inv_t, sizeof(T) == 4 ? fmaf(fmaxf(acc[j][i][x], -1e30f), a.inv_lo, -lse) : -lse),
                    p = __expf(logp);
        acc[j][i][x] = -p * (g + e * (fmaxf(logp, -1e30f) + H));
      }
    const int tcol = y >= 0 ? y - col0 : -1;
    if (__ballot((unsigned)tcol < 64u)) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[j][i][x] += pt_col(j, x, hf) == tcol ? g : 0.f;
    }
  }
  const bool edge = a.V - col0 < 64 || row0 + 32 * MT > a.T;  // some of the wave's columns or rows do not exist: zeros
  char* const ep = PT_WAVE_LDS;
  T* const dz = (T*)a.dz + (size_t)row0 * a.ldz + col0;
  if constexpr (sizeof(T) == 2) {
    pt_hand_out<8, MT>(ep, lane, acc, PtNothing(), [&](int r, int c, float(&v)[8], int) {
      if (edge) {
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = row0 + r < a.T && col0 + c + u < a.V ? v[u] : 0.f;
      }
      if (row0 + r < a.rows) *(pt_u32x4*)(dz + (size_t)r * a.ldz + c) = pt_pack8<T>(v);
    });
  } else {
    pt_hand_out<4, MT>(ep, lane, acc, PtNothing(), [&](int r, int c, pt_f32x4 v, int) {
      if (edge) {
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = row0 + r < a.T && col0 + c + u < a.V ? v[u] : 0.f;
      }
      if (row0 + r < a.rows) *(pt_f32x4*)(dz + (size_t)r * a.ldz + c) = v;
    });
  }
}

// out [M, N] (T or float) = scale * A W', or the fp32 slabs of a product cut along K.  dz of 13,568 x 50,304 in bfloat16, d = 2,560: dh 2.9 ms
// (1,200 TFLOP/s, and 0.17 for the sum of six slabs), dW 2.8 (1,250): matrix products, near what the library's reach.
struct OutArgs {
  const void *A, *W, *w_end;  // (see pt_product)
  uint32_t lda, ldw;
  int M, N, K, slices, k_slice;
  const float* scale;  // null: 1
  void* out;
  size_t ldo;
  int f32, add;  // out is float; added to what is there (float only)
  float* slab;   // slices > 1: [slice][M][lds]
  int lds, tile0, tiles_n;
};

template <typename T>
__device__ __forceinline__ void out_store(const OutArgs& a, int row, int col, pt_f32x4 v, bool vec) {
  if (a.slices > 1) return;
  if (a.f32) {
    float* const o = (float*)a.out + (size_t)row * a.ldo + col;
    if (vec && col + 4 <= a.N) {
      if (a.add) v += *(const pt_f32x4*)o;
      *(pt_f32x4*)o = v;
    } else {
      for (int u = 0; u < 4; ++u)
        if (col + u < a.N) o[u] = a.add ? o[u] + v[u] : v[u];
    }
  } else {
    T* const o = (T*)a.out + (size_t)row * a.ldo + col;
    for (int u = 0; u < 4; ++u)
      if (col + u < a.N) o[u] = (T)v[u];
  }
}

template <typename T, bool AK, bool WK, typename S>
__global__ void __launch_bounds__(64 * S::waves, pt_waves_eu<S>) out_kernel(OutArgs a) {
  PT_STAGES(S)
  constexpr int MT = S::MT;
  // (rows are walked as columns are elsewhere: dW has many of them, dh is cut along K)
  const int nb_m = a.tiles_n, nb_n = (a.N + S::cols - 1) / S::cols;
  const int item = pt_item_rounds(nb_m * nb_n * a.slices);
  if (item < 0) return;
  const int z = item / (nb_m * nb_n);
  int tm, tn;
  pt_tile_pos(item - z * nb_m * nb_n, nb_m, nb_n, tm, tn);
  tm += a.tile0;
  pt_f32x16 acc[2][MT];
  const int k1 = min(a.K, (z + 1) * a.k_slice);
  PT_PRODUCT(T, AK, WK, a.A, a.lda, tm * S::rows, a.M, a.W, a.ldw, tn * S::cols, a.N, z * a.k_slice, k1, k1 == a.K ? a.w_end : nullptr);
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (pt_done<S>(wave)) return;
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
  char* const ep = PT_WAVE_LDS;
  if (a.slices > 1) {
    float* const o = a.slab + (size_t)z * a.M * a.lds;
    pt_hand_out<4, MT>(ep, lane, acc, PtNothing(), [&](int r, int c, pt_f32x4 v, int) {
      if (row0 + r < a.M && col0 + c < a.lds) *(pt_f32x4*)(o + (size_t)(row0 + r) * a.lds + col0 + c) = v;
    });
    return;
  }
  const float s = a.scale ? a.scale[1] : 1.f;
  const bool vec = ((uintptr_t)a.out & 15) == 0 && a.ldo % (a.f32 ? 4 : 8) == 0;
  if (sizeof(T) == 2 && !a.f32) {
    if constexpr (sizeof(T) == 2) {
      pt_hand_out<8, MT>(ep, lane, acc, PtNothing(), [&](int r, int c, float(&v)[8], int) {
        if (row0 + r >= a.M) return;
        T* const o = (T*)a.out + (size_t)(row0 + r) * a.ldo + col0 + c;
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] *= s;
        if (vec && col0 + c + 8 <= a.N) {
          *(pt_u32x4*)o = pt_pack8<T>(v);
        } else {
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (col0 + c + u < a.N) o[u] = (T)v[u];
        }
      });
    }
  } else {
    pt_hand_out<4, MT>(ep, lane, acc, PtNothing(), [&](int r, int c, pt_f32x4 v, int) {
      if (row0 + r < a.M) out_store<T>(a, row0 + r, col0 + c, v * s, vec);
    });
  }
}

// out = scale * the sum of the slabs in their order
template <typename T>
__global__ void __launch_bounds__(256) out_sum_kernel(OutArgs a) {
  const int quads = a.lds / 4;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)a.M * quads) return;
  const int row = (int)(i / quads), col = (int)(i - (size_t)row * quads) * 4;
  const float* const p = a.slab + (size_t)row * a.lds + col;
  pt_f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int z0 = 0; z0 < a.slices; z0 += 8) {  // (eight loads under way)
    pt_f32x4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = *(const pt_f32x4*)(p + (size_t)min(z0 + k, a.slices - 1) * a.M * a.lds);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (z0 + k < a.slices) v += x[k];
  }
  const float s = a.scale ? a.scale[1] : 1.f;
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] *= s;
  a.slices = 1;
  out_store<T>(a, row, col, v, ((uintptr_t)a.out & 15) == 0 && a.ldo % 4 == 0);
}

// out (T) = a (float), n elements
template <typename T>
__global__ void __launch_bounds__(256) narrow_rows_kernel(const float* __restrict__ a, int cols, T* __restrict__ out, size_t ldo) {
  for (int c = threadIdx.x; c < cols; c += 256) out[(size_t)blockIdx.x * ldo + c] = (T)a[(size_t)blockIdx.x * cols + c];
}

int tiles(int m, int n, int tm, int tn) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); }

size_t elem_size(int dtype) { return dtype == kTokensF32 ? 4 : 2; }
int stage_of(int dtype) { return 128 / (int)elem_size(dtype); }  // k of a stage of the products
int whole(int n, int stage) { return (n + stage - 1) / stage * stage; }
int padded(int n) { return whole(n, 64); }

// How a product's columns are cut: `big` column tiles of 256 (256 x 256, a CU each) first, the rest in tiles of 128 (128 x 128, two
// on a CU).  16-bit types: a round of 256 large tiles takes 1.95 us a stage, one of 512 small ones 1.5 (and of up to 256 1.0), so
// the large ones make whole rounds and the small ones what is left.  float: the matrix instructions take 16 times as long and
// nothing else counts: per tile as much as its area.
int big_columns(int M, int N, int dtype, double* takes = nullptr) {
  const int nb_m = (M + 255) / 256, nb_n = (N + 255) / 256, mid_m = (M + 127) / 128, mid_n = (N + 127) / 128;
  const double round = dtype == kTokensF32 ? 4.0 : 1.95, small = dtype == kTokensF32 ? 2.0 : 1.5, half = dtype == kTokensF32 ? 1.05 : 1.0;
  auto cost = [&](int n) {
    const int rest = mid_m * std::max(0, mid_n - 2 * n);
    const double mids = rest == 0 ? 0.0 : rest % 512 == 0 ? rest / 512 * small : rest / 512 * small + (rest % 512 <= 256 ? half : small);
    return (double)((nb_m * n + 255) / 256) * round + mids + (n > 0 && rest > 0 ? 0.2 : 0.0);
  };
  int best = 0;
  double best_c = cost(0);
  for (int r = (nb_m * nb_n + 255) / 256; r > 0; --r) {  // (the most that r rounds hold)
    const int n = std::min(nb_n, 256 * r / nb_m);
    if (n > 0 && cost(n) < best_c - 1e-9) best = n, best_c = cost(n);
  }
  if (takes) *takes = best_c;
  return best;
}
// Or, float, 32 x 64, whose four waves share a tile's K: for few rows, whose tiles would be mostly empty, and for few tiles.  (K = 4,096: one
// row of 50,304 495 -> 197 us, of 1,000 264 -> 63; 106 rows of 50,304, K = 512, the gradient, 216 -> 226, which the rule leaves.  16-bit
// types wait for W: 64 rows, K = 2,560, 77 -> 94.)
constexpr double kThinStart = 6;  // stages that a tile's start and end take
double thin_cost(int n, int dtype) { return dtype == kTokensF32 ? 0.15 * ((n + 255) / 256) : 1e9; }
bool thin(int M, int N, int K, int dtype) {
  double wide;
  big_columns(M, N, dtype, &wide);
  const int stages = (K + stage_of(dtype) - 1) / stage_of(dtype);
  return thin_cost(tiles(M, N, 32, 64), dtype) * (stages + kThinStart) < wide * (stages + 1.5);
}

struct Bump {
  char* base;
  size_t off = 0;
  template <typename T>
  T* take(size_t n) {
    off = (off + 255) & ~(size_t)255;
    T* const p = base ? (T*)(base + off) : nullptr;
    off += n * sizeof(T);
    return p;
  }
};

constexpr int kLogitRows = 16384;  // rows of stored logits at a time
constexpr int kSumRows = 65536;    // rows at a time where none are: a launch's threads stay below 2^32, the parts' sums at 0.6 GB
constexpr int kGradRows = 16384;   // rows of dz at a time

int equal_chunk(int T, int most) {  // rows of a chunk: as few chunks as there must be, of about the same size
  const int n = (T + most - 1) / most;
  return std::min(T, ((T + n - 1) / n + 255) & ~255);
}

template <typename F>
void by_type(int dtype, F f) {
  if (dtype == kTokensF32) f(float());
  else if (dtype == kTokensBF16) f(bfloat());
  else f(half_t());
}

struct Operand {
  const void *p, *end;  // end: the last rows, up to a whole stage of them, where they are summed over and are not one
  uint32_t ld;
};
// The matrix as the products read it: as it lies, or a copy in the workspace with zeros up to whole stages (a null workspace: measuring).
// Where its rows are summed over and it ends inside a stage, that stage alone is copied.
Operand packed(Bump& ws, const TokenRows& m, int rows, int d, int dtype, bool rows_as_k, hipStream_t s) {
  auto copy = [&](int from, int n, int ldd, int rows_to) {
    char* const to = ws.take<char>((size_t)rows_to * ldd * elem_size(dtype));
    if (to)
      by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const size_t chunks = (size_t)rows_to * ldd / (16 / sizeof(T));
        hipLaunchKernelGGL(pack_rows_kernel<T>, dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, s, (const T*)m.p + (size_t)from * m.ld,
                           (size_t)m.ld, n, d, (T*)to, ldd, rows_to);
      });
    return to;
  };
  if (!m.lies_well) return {copy(0, rows, padded(d), padded(rows)), nullptr, (uint32_t)padded(d)};
  const int stage = stage_of(dtype), over = rows % stage;
  return {m.p, rows_as_k && over ? copy(rows - over, over, (int)m.ld, stage) : nullptr, (uint32_t)m.ld};
}

size_t finish_lds(int parts, int rows, int top) {
  return top ? ((size_t)rows * (parts | 1) + (size_t)std::min(rows, 4) * finish_words(top)) * 4 : 0;
}

// Column tiles of 256 whose logits are stored whole, so that their part maxima bound what the others need to store; 0: one launch
// that stores all.  The shortest of rounds of tiles (see big_columns) times K's stages, what is stored at 5 TB/s (parts by
// themselves at half of it), and 7 us for the bound and its launch.  (13,568 rows of 50,304 entries, K = 2,560, eight alternatives:
// all stored 3.33 ms, this way 2.89, no alternatives 2.74; 1,003 rows of 50,277, K = 1,037, five: 203 and 196 us; 2,000 of 50,304,
// K = 768, eight: 269 and 234.)
int sample_tiles(int T, int V, int K, int top, int dtype) {
  const int nb_n = (V + 255) / 256;
  double all;
  if (!top || !big_columns(T, V, dtype, &all)) return 0;
  const double stage = (dtype == kTokensF32 ? 2.0 : 1.0) * ((K + stage_of(dtype) - 1) / stage_of(dtype) + 4), column = 256.0 * T * 4 / 5e6;
  int best = 0;
  double best_t = all * stage + nb_n * column;
  for (int n = top; n <= std::min(nb_n / 2, 239); ++n) {  // (stats_threshold_kernel holds 16 rows of 4 n maxima in 60 KB)
    double rest;
    big_columns(T, V - 256 * n, dtype, &rest);
    const double rounds = (((T + 255) / 256) * n + 255) / 256 * (dtype == kTokensF32 ? 4.0 : 1.95);
    const double kept = (nb_n - n) * column * std::min(1.0, top / (4.0 * n));  // parts that the bound does not rule out
    const double t = (rounds + rest) * stage + n * column + 2 * kept + 7;
    if (t < best_t) best = n, best_t = t;
  }
  return best;
}

}  // namespace

bool token_rows_lie_well(int64_t ld, int d, int dtype, int rows_as_k) {
  return ld % (16 / (int)elem_size(dtype)) == 0 && d % stage_of(dtype) == 0 && (rows_as_k % stage_of(dtype) == 0 || ld <= 1 << 16);
}

size_t token_stats_plan(const TokenStatsArgs& a, void* workspace, hipStream_t s, hipError_t* err) {
  Bump ws{(char*)workspace};
  const int parts = (a.V + kPart - 1) / kPart;
  const Operand h = packed(ws, a.hidden, a.T, a.d, a.dtype, false, s), w = packed(ws, a.weight, a.V, a.d, a.dtype, false, s);
  const int rows = equal_chunk(a.T, a.top ? kLogitRows : kSumRows);
  StatsArgs k;
  float* const part = ws.take<float>((size_t)3 * parts * rows);
  float* const ztgt = ws.take<float>(rows);
  float* const thr = ws.take<float>(a.top ? rows : 0);
  float* const logits = a.top ? ws.take<float>((size_t)rows * padded(a.V)) : nullptr;
  if (!workspace) return ws.off;
  for (int t0 = 0; t0 < a.T; t0 += rows) {
    const int n = std::min(rows, a.T - t0);
    k.h = (const char*)h.p + (size_t)t0 * h.ld * elem_size(a.dtype);
    k.w = w.p;
    k.ldh = h.ld;
    k.ldw = w.ld;
    k.T = n;
    k.V = a.V;
    k.d = whole(a.d, stage_of(a.dtype));
    k.targets = a.targets + t0;
    k.inv_t = a.inv_t;
    k.pmax = part;
    k.ps0 = part + (size_t)parts * n;
    k.ps1 = k.ps0 + (size_t)parts * n;
    k.ztgt = ztgt;
    k.logits = logits;
    k.ldl = padded(a.V);
    k.thr = nullptr;
    by_type(a.dtype, [&](auto t) {
      using T = decltype(t);
      auto run = [&](auto shape, int from, int to) {
        using S = decltype(shape);
        k.tile0 = from;
        k.tiles_n = to - from;
        hipLaunchKernelGGL((stats_kernel<T, S>), dim3(pt_grid(((n + S::rows - 1) / S::rows) * (to - from))), dim3(64 * S::waves), 0, s, k);
      };
      const int big = big_columns(n, a.V, a.dtype), mids = (a.V + 127) / 128;
      if (const int first = sample_tiles(n, a.V, a.d, a.top, a.dtype)) {
        run(PtBig(), 0, first);
        hipLaunchKernelGGL(stats_threshold_kernel, dim3(pt_grid((n + 15) / 16)), dim3(256), 16 * (size_t)(4 * first | 1) * 4, s, k.pmax, n, 4 * first,
                           a.top, thr);
        k.thr = thr;
        const int then = first + big_columns(n, a.V - 256 * first, a.dtype);
        if (then > first) run(PtBig(), first, then);
        if (2 * then < mids) run(PtMid(), 2 * then, mids);
      } else {
        bool done = false;
        if constexpr (sizeof(T) == 4) {
          if ((done = thin(n, a.V, a.d, a.dtype))) run(PtThin(), 0, parts);
        }
        if (!done && big) run(PtBig(), 0, big);
        if (!done && 2 * big < mids) run(PtMid(), 2 * big, mids);
      }
    });
    FinishArgs f = {k.pmax, k.ps0, k.ps1, ztgt, logits, k.targets, n, a.V, parts, k.ldl, a.top, a.inv_t, a.inv_lo,
                    a.logprob + t0, a.entropy + t0, a.lse + t0, a.top ? a.top_ids + (size_t)t0 * a.top : nullptr,
                    a.top ? a.top_logprob + (size_t)t0 * a.top : nullptr};
    auto finish = [&](auto r) {
      constexpr int R = decltype(r)::value;
      hipLaunchKernelGGL(stats_finish_kernel<R>, dim3(pt_grid((n + R - 1) / R)), dim3(256), finish_lds(parts, R, a.top), s, f);
    };
    // rows of a finishing block: many share the lines of the parts' sums, few leave no CU idle
    if (n >= 4096 && finish_lds(parts, 8, a.top) <= 60 * 1024) finish(std::integral_constant<int, 8>{});
    else if (n >= 512 && finish_lds(parts, 4, a.top) <= 60 * 1024) finish(std::integral_constant<int, 4>{});
    else finish(std::integral_constant<int, 1>{});
    if ((*err = hipGetLastError()) != hipSuccess) return ws.off;
  }
  return ws.off;
}

// The slices of K of a product, and the row tiles of 256 that go first (see big_columns; the rest has none).  Few tiles over a long K
// are cut along it: as many slices as make rounds times a slice's length shortest, each at least 512 long, with what the fp32
// slabs cost to write and to read again (5 TB/s).
struct OutPlan {
  int slices, k_slice, big, thin;
};
static OutPlan out_plan(int M, int N, int K, int dtype) {
  const int stage = stage_of(dtype);
  OutPlan best = {1, K, 0, 0};
  double best_t = 1e30;
  for (int z = 1; z <= 64; ++z) {
    const int q = whole((K + z - 1) / z, stage);
    if (z > 1 && (q < 512 || (K + q - 1) / q != z)) continue;
    const double us = dtype == kTokensF32 ? 2.0 : 1.0;  // of a stage, in big_columns' units
    const double slabs = z > 1 ? z * ((double)M * N * 8 / 5e6) + 4 : 0;
    for (int big = 0; big < 3; ++big) {
      const int n = big == 2 ? tiles(M, N, 32, 64) * z : big ? tiles(M, N, 256, 256) * z : tiles(M, N, 128, 128) * z;
      const double rounds = big == 2 ? thin_cost(n, dtype) : big ? std::ceil(n / 256.0) * (dtype == kTokensF32 ? 4.0 : 1.95)
                                : n / 512 * (dtype == kTokensF32 ? 2.0 : 1.5) + (n % 512 == 0 ? 0.0 : n % 512 <= 256 ? 1.0 : dtype == kTokensF32 ? 2.0 : 1.5);
      const double t = rounds * us * (q / stage + (big == 2 ? kThinStart : dtype == kTokensF32 ? 1.5 : 3.0)) + slabs;
      if (t < best_t) best_t = t, best = {z, q, big == 1 ? (M + 255) / 256 : 0, big == 2};
    }
  }
  if (best.slices == 1 && !best.thin) best.big = big_columns(N, M, dtype);
  return best;
}

template <typename T, bool AK, bool WK>
static void launch_out(OutArgs& o, const OutPlan& p, hipStream_t s) {
  auto run = [&](auto shape, int from, int to) {
    using S = decltype(shape);
    o.tile0 = from;
    o.tiles_n = to - from;
    const int n = (to - from) * ((o.N + S::cols - 1) / S::cols) * o.slices;
    hipLaunchKernelGGL((out_kernel<T, AK, WK, S>), dim3(pt_grid(n)), dim3(64 * S::waves), 0, s, o);
  };
  const int mids = (o.M + 127) / 128;
  if constexpr (sizeof(T) == 4) {
    if (p.thin) run(PtThin(), 0, (o.M + 31) / 32);
  }
  if (p.big) run(PtBig(), 0, p.big);
  if (!p.thin && 2 * p.big < mids) run(PtMid(), 2 * p.big, mids);
  if (o.slices > 1) {
    const size_t n = (size_t)o.M * (o.lds / 4);
    hipLaunchKernelGGL(out_sum_kernel<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, o);
  }
}

size_t token_stats_backward_plan(const TokenGradArgs& a, void* workspace, hipStream_t s, hipError_t* err) {
  Bump ws{(char*)workspace};
  const Operand h = packed(ws, a.hidden, a.T, a.d, a.dtype, true, s), w = packed(ws, a.weight, a.V, a.d, a.dtype, true, s);
  const int esz = (int)elem_size(a.dtype), stage = stage_of(a.dtype), rows = equal_chunk(a.T, kGradRows);
  const int ldz = padded(a.V), kv = whole(a.V, stage), lds = (a.d + 3) & ~3;
  const bool chunks = rows < a.T;
  float* const scale = ws.take<float>(2);
  char* const dz = ws.take<char>((size_t)whole(rows, stage) * ldz * esz);
  // sums over several chunks of rows are formed in fp32: in the output, or here
  const bool grads_f32 = a.grad_f32 || a.dtype == kTokensF32;
  float* const dw32 = chunks && !grads_f32 ? ws.take<float>((size_t)a.V * a.d) : nullptr;
  size_t slab = 0;
  for (int t0 = 0; t0 < a.T; t0 += rows) {
    const int n = std::min(rows, a.T - t0);
    const int zh = out_plan(n, a.d, kv, a.dtype).slices, zw = out_plan(a.V, a.d, whole(n, stage), a.dtype).slices;
    slab = std::max(slab, std::max(zh > 1 ? (size_t)zh * n * lds : 0, zw > 1 ? (size_t)zw * a.V * lds : 0));
  }
  float* const slabs = ws.take<float>(slab);
  if (!workspace) return ws.off;
  const bool scaled = a.dtype == kTokensF16;
  if (scaled)
    hipLaunchKernelGGL(grad_scale_kernel, dim3(1), dim3(1024), 0, s, a.targets, a.d_logprob, a.d_entropy, a.T, a.V, a.inv_t, scale);
  for (int t0 = 0; t0 < a.T; t0 += rows) {
    const int n = std::min(rows, a.T - t0);
    const void* const hp = (const char*)h.p + (size_t)t0 * h.ld * esz;
    DzArgs k = {hp, w.p, h.ld, w.ld, n, a.V, whole(a.d, stage), a.targets + t0, a.lse + t0, (a.d_entropy ? a.entropy : a.lse) + t0, a.d_logprob + t0,
                      a.d_entropy ? a.d_entropy + t0 : nullptr, scaled ? scale : nullptr, a.inv_t, a.inv_lo, dz, ldz, whole(n, stage), 0, 0};
    OutArgs oh = {}, ow = {};
    oh.A = dz;
    oh.lda = ldz;
    oh.W = w.p;
    oh.ldw = w.ld;
    oh.w_end = w.end;
    oh.M = n;
    oh.N = a.d;
    oh.K = kv;
    const OutPlan ph = out_plan(n, a.d, kv, a.dtype);
    oh.slices = ph.slices;
    oh.k_slice = ph.k_slice;
    oh.out = (char*)a.d_hidden + (size_t)t0 * a.d * (grads_f32 ? 4 : 2);
    oh.ldo = a.d;
    oh.f32 = grads_f32;
    ow.A = dz;
    ow.lda = ldz;
    ow.W = hp;
    ow.ldw = h.ld;
    ow.w_end = n % stage ? h.end : nullptr;  // (the last rows')
    ow.M = a.V;
    ow.N = a.d;
    ow.K = whole(n, stage);
    const OutPlan pw = out_plan(a.V, a.d, ow.K, a.dtype);
    ow.slices = pw.slices;
    ow.k_slice = pw.k_slice;
    ow.out = dw32 ? (void*)dw32 : a.d_weight;
    ow.ldo = a.d;
    ow.f32 = grads_f32 || dw32;
    ow.add = t0 > 0;
    oh.scale = ow.scale = scaled ? scale : nullptr;
    oh.slab = ow.slab = slabs;
    oh.lds = ow.lds = lds;
    by_type(a.dtype, [&](auto t) {
      using T = decltype(t);
      auto run = [&](auto shape, int from, int to) {
        using S = decltype(shape);
        k.tile0 = from;
        k.tiles_n = to - from;
        hipLaunchKernelGGL((dz_kernel<T, S>), dim3(pt_grid(((n + S::rows - 1) / S::rows) * (to - from))), dim3(64 * S::waves), 0, s, k);
      };
      const int big = big_columns(n, a.V, a.dtype), mids = (a.V + 127) / 128;
      bool done = false;
      if constexpr (sizeof(T) == 4) {
        if ((done = thin(n, a.V, a.d, a.dtype))) run(PtThin(), 0, ldz / 64);
      }
      if (!done && big) run(PtBig(), 0, big);
      if (!done && 2 * big < mids) run(PtMid(), 2 * big, mids);
      launch_out<T, false, true>(oh, ph, s);
      launch_out<T, true, true>(ow, pw, s);
    });
    if ((*err = hipGetLastError()) != hipSuccess) return ws.off;
  }
  if (dw32)
    by_type(a.dtype, [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL(narrow_rows_kernel<T>, dim3(a.V), dim3(256), 0, s, (const float*)dw32, a.d, (T*)a.d_weight, (size_t)a.d);
    });
  *err = hipGetLastError();
  return ws.off;
}

}  // namespace rlhf
