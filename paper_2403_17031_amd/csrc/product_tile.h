// Tiles of matrix products for the operators of an update (token_stats.hip, muon.hip): C[M,N] = sum_k A(m,k) W(n,k), in half,
// bfloat16 or float, with an epilogue of the caller's, several products in one launch.
//
// Either operand is row-major (its rows hold k: a [M, K] or [N, K] matrix) or K-major ([K, M] or [K, N], so that a product
// with a transposed matrix reads the matrix as it lies).  A stage is 128 bytes of k per row (64 k of 16-bit types, 32 of float),
// brought from global memory straight to LDS; two stages alternate.  Row-major stages hold rows of 128 bytes whose
// eight 16-byte chunks are XORed with bits 1..3 of the row, so that the 32 rows of an operand slice are read without
// bank conflicts; K-major stages hold k-rows, chunk c of k-row k at c ^ 2(k mod 4), and 16-bit slices come from the
// transposing LDS read (two of four k each).
//
// The loads of a stage are issued while the last quarter of the stage before it is multiplied and have a whole stage to
// land; fragments of a quarter stage are read while the quarter before is multiplied.
//
// Rows past M or N repeat the last one and are not stored.  K is whole stages: operands that are not lie in
// the caller's workspace with zeros up to there.  Row strides and bases are whole 16-byte chunks.
#pragma once
#include <type_traits>

#include "common.h"

namespace rlhf {

typedef __attribute__((ext_vector_type(16))) float pt_f32x16;
typedef __attribute__((ext_vector_type(4))) float pt_f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t pt_u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t pt_u32x2;
typedef __attribute__((ext_vector_type(8))) _Float16 pt_f16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 pt_bf16x8;
typedef __bf16 bfloat;

// c += the outer products of two operand slices (16 bytes a lane: k = 16-byte chunk `lane / 32` of a pair of chunks)
__device__ __forceinline__ pt_f32x16 pt_mma(half_t, pt_u32x4 w, pt_u32x4 a, pt_f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(pt_f16x8, w), __builtin_bit_cast(pt_f16x8, a), c, 0, 0, 0);
}
__device__ __forceinline__ pt_f32x16 pt_mma(bfloat, pt_u32x4 w, pt_u32x4 a, pt_f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pt_bf16x8, w), __builtin_bit_cast(pt_bf16x8, a), c, 0, 0, 0);
}
__device__ __forceinline__ pt_f32x16 pt_mma(float, pt_u32x4 w, pt_u32x4 a, pt_f32x16 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[e]), __uint_as_float(a[e]), c, 0, 0, 0);
  return c;
}

#define PT_GLOBAL(p) ((const __attribute__((address_space(1))) void*)(p))
#define PT_LDS(p) ((__attribute__((address_space(3))) void*)(p))

#define PT_WAVE_LDS_FENCE()                          \
  __builtin_amdgcn_sched_barrier(0);                 \
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); \
  __builtin_amdgcn_wave_barrier();                   \
  __builtin_amdgcn_sched_barrier(0);

// WM x WN waves of MT x NT accumulators of 32 x 32; RING stages of LDS (2: see pt_product, more: pt_product_ring); KW such sets of
// waves, each with its quarter of every stage (4, or 1).
template <int WM_, int WN_, int MT_, int NT_, int RING_ = 2, int KW_ = 1>
struct PtShape {
  static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = NT_, RING = RING_, KW = KW_;
  static constexpr int waves = WM * WN * KW, rows = 32 * MT * WM, cols = 32 * NT * WN, stage = (rows + cols) * 128;
  static_assert(KW == 1 || (KW == 4 && RING > 2 && 3 * WM * WN * MT * NT * 4096 <= RING * stage), "quarters, their sums in the ring");
};

// One operand's tile loads: this lane's 16-byte chunks of a stage, as byte offsets from a uniform base.
template <typename T, bool KM, int ROWS, int NW>
struct PtLoads {
  static constexpr int E = 16 / (int)sizeof(T), KD = 128 / (int)sizeof(T), L = ROWS / (8 * NW);
  static constexpr int RB = KM ? ROWS * (int)sizeof(T) : 128;  // bytes of a stage's LDS row
  const char* base;
  const char* end = nullptr;  // where the stage `at_end` lies instead
  int at_end = -1;
  uint32_t off[L];
  size_t step;

  __device__ static int lds_row(int i, int wave, int lane) { return (1024 * (L * wave + i) + 16 * lane) / RB; }
  __device__ static int chunk(int i, int wave, int lane) {
    const int r = lds_row(i, wave, lane), pos = ((1024 * (L * wave + i) + 16 * lane) % RB) / 16;
    return KM ? pos ^ (2 * (r & 3)) : pos ^ ((r >> 1) & 7);
  }
  __device__ __forceinline__ const char* stage_at(int stage) const { return KM && stage == at_end ? end : base + stage * step; }
  // the same through load_to_lds, for a caller that counts its waits
  __device__ __forceinline__ void load_counted(uint32_t lds, int stage, int i, int wave) const {
    load_to_lds(stage_at(stage), off[i], lds + 1024 * (L * wave + i));
  }
  // the operand from its row r0 (of `extent`) on, from k0 on
  __device__ void init(const void* p, uint32_t ld, int r0, int extent, int k0, int wave, int lane) {
    const size_t stride = (size_t)ld * sizeof(T);
    base = (const char*)p + (KM ? (size_t)k0 * stride + (size_t)r0 * sizeof(T) : (size_t)r0 * stride + (size_t)k0 * sizeof(T));
    step = KM ? KD * stride : 128;
    const int left = extent - r0;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int r = lds_row(i, wave, lane), c = chunk(i, wave, lane);
      off[i] = KM ? (uint32_t)(r * stride) + 16u * (uint32_t)min(c, (left - 1) / E)
                  : (uint32_t)(min(r, left - 1) * stride) + 16u * (uint32_t)c;
    }
  }
  __device__ __forceinline__ void load(char* lds, int stage, int i, int wave) const {
    const char* p = stage_at(stage);
    asm volatile("" : "+s"(p));  // (uniform: a scalar base and the lane's 32-bit offset)
    uint32_t o = off[i];
    asm volatile("" : "+v"(o));
    __builtin_amdgcn_global_load_lds(PT_GLOBAL(p + o), PT_LDS(lds + 1024 * (L * wave + i)), 16, 0, 0);
  }
};

// Reads of an operand slice: 32 rows from row0 on, quarter stage s.
template <typename T, bool KM, int ROWS>
struct PtFrags {
  static constexpr int RB = KM ? ROWS * (int)sizeof(T) : 128;
  int at;
  __device__ void init(int row0, int lane) {
    const int l32 = lane & 31, hf = lane >> 5;
    if constexpr (!KM) {
      at = (row0 + l32) * 128;
    } else if constexpr (sizeof(T) == 2) {
      const int r = lane & 15, colb = row0 + 16 * ((lane >> 4) & 1);
      const int c = ((colb >> 3) + ((r & 3) >> 1)) ^ (2 * ((r >> 2) & 3));
      at = (8 * hf + (r >> 2)) * RB + c * 16 + (r & 1) * 8;
    } else {
      at = row0 + l32;  // column
    }
  }
  __device__ __forceinline__ pt_u32x4 read(const char* lds, int s, int lane) const {
    const int hf = lane >> 5;
    if constexpr (!KM) {
      const int key = ((lane & 31) >> 1) & 7;
      return *(const pt_u32x4*)(lds + at + (((2 * s + hf) ^ key) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((ext_vector_type(4))) short s16x4;
      typedef __attribute__((address_space(3))) s16x4* lds4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(lds + at + 16 * s * RB));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(lds + at + (16 * s + 4) * RB));
      const pt_u32x2 l = __builtin_bit_cast(pt_u32x2, lo), h = __builtin_bit_cast(pt_u32x2, hi);
      return pt_u32x4{l[0], l[1], h[0], h[1]};
    } else {
      pt_u32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int k = 8 * s + 4 * hf + e;
        v[e] = *(const uint32_t*)(lds + k * RB + (((at >> 2) ^ (2 * (k & 3))) << 4) + (at & 3) * 4);
      }
      return v;
    }
  }
};

// acc = the product over k0 <= k < k1 of one tile; la*, lw*: the stages' LDS (separate variables, so that a read of one stage does not
// wait for the loads into the other).  k1 - k0 is a positive multiple of a stage's depth.  w_end: the last stage of a K-major W lies
// there, with W's row stride, where W itself ends inside of it; or null.
template <typename T, bool AK, bool WK, typename S>
__device__ __forceinline__ void pt_product(const void* A, uint32_t lda, int m0, int M, const void* W, uint32_t ldw, int n0, int N,
                                           int k0, int k1, const void* w_end, char* la0, char* lw0, char* la1, char* lw1,
                                           pt_f32x16 (&acc)[S::NT][S::MT]) {
  constexpr int MT = S::MT, NT = S::NT, F = MT + NT, NMF = MT * NT;
  using LA = PtLoads<T, AK, S::rows, S::waves>;
  using LW = PtLoads<T, WK, S::cols, S::waves>;
  constexpr int NL = LA::L + LW::L;
  constexpr int STEPS = NMF > F ? (NMF > NL ? NMF : NL) : (F > NL ? F : NL);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / S::WN) * 32 * MT, wn = (wave % S::WN) * 32 * NT;
  LA ga;
  LW gw;
  ga.init(A, lda, m0, M, k0, wave, lane);
  gw.init(W, ldw, n0, N, k0, wave, lane);
  PtFrags<T, AK, S::rows> ra[MT];
  PtFrags<T, WK, S::cols> rw[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) ra[i].init(wm + 32 * i, lane);
#pragma unroll
  for (int j = 0; j < NT; ++j) rw[j].init(wn + 32 * j, lane);
  const int nk = (k1 - k0) / LA::KD;
  if (WK && w_end) {
    gw.end = (const char*)w_end + (size_t)n0 * sizeof(T);
    gw.at_end = nk - 1;
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;
  auto load_one = [&](char* la, char* lw, int stage, int n) {
    if (n < LA::L) ga.load(la, stage, n, wave);
    else gw.load(lw, stage, n - LA::L, wave);
  };
  auto load_all = [&](char* la, char* lw, int stage) {
#pragma unroll
    for (int n = 0; n < NL; ++n) load_one(la, lw, stage, n);
  };
  pt_u32x4 fa[2][MT], fw[2][NT];
  auto frag = [&](const char* la, const char* lw, int s, int n, int buf) {
    if (n < MT) fa[buf][n] = ra[n].read(la, s, lane);
    else fw[buf][n - MT] = rw[n - MT].read(lw, s, lane);
  };
  // a quarter stage: the matrix instructions on fragments `buf`; between them the next quarter's fragment reads and, if LOAD,
  // the tile loads of a later stage
  auto sub = [&](int buf, const char* la, const char* lw, int s, auto load, char* da, char* dw, int stage) {
    constexpr bool LOAD = decltype(load)::value;
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
      if (n < NMF) {
        const int j = n / MT, i = (j & 1) ? MT - 1 - n % MT : n % MT;  // serpentine: one operand changes at a time
        acc[j][i] = pt_mma(T(), fw[buf][j], fa[buf][i], acc[j][i]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (n < F) frag(la, lw, s, n, buf ^ 1);
      if (LOAD && n < NL && stage < nk) load_one(da, dw, stage, n);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  using No = std::false_type;
  using Yes = std::true_type;
  // every wave's tile loads have landed and every wave has finished reading the current stage
  auto wait = [&] {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // stage kt in (ca, cw); the next one is landing in (oa, ow)
  auto stage = [&](int kt, char* ca, char* cw, char* oa, char* ow) {
    sub(0, ca, cw, 1, No(), nullptr, nullptr, 0);
    sub(1, ca, cw, 2, No(), nullptr, nullptr, 0);
    sub(0, ca, cw, 3, No(), nullptr, nullptr, 0);
    wait();
    sub(1, oa, ow, 0, Yes(), ca, cw, kt + 2);  // (the last stage's fragments are of nothing, and not used)
  };
  load_all(la0, lw0, 0);
  if (nk > 1) load_all(la1, lw1, 1);
  wait();
#pragma unroll
  for (int n = 0; n < F; ++n) frag(la0, lw0, 0, n, 0);
  int kt = 0;
  for (; kt + 1 < nk; kt += 2) {
    stage(kt, la0, lw0, la1, lw1);
    stage(kt + 1, la1, lw1, la0, lw0);
  }
  if (kt < nk) stage(kt, la0, lw0, la1, lw1);
}

// The same with a ring of S::RING stages, all but one of them under way while one is used: for launches whose tiles do not fill
// the chip, where a stage's loads take longer than its multiplications.  The compiler does not know of the loads; what orders
// them is the counted wait before the barrier.  Ends as pt_product does; with quarters, the first set of waves has the sums
// and the others are done (pt_done).
template <typename T, bool AK, bool WK, typename S>
__device__ __forceinline__ void pt_product_ring(const void* A, uint32_t lda, int m0, int M, const void* W, uint32_t ldw, int n0, int N,
                                                int k0, int k1, const void* w_end, char* lds, pt_f32x16 (&acc)[S::NT][S::MT]) {
  constexpr int MT = S::MT, NT = S::NT, F = MT + NT, D = S::RING;
  using LA = PtLoads<T, AK, S::rows, S::waves>;
  using LW = PtLoads<T, WK, S::cols, S::waves>;
  constexpr int NL = LA::L + LW::L;
  static_assert((D - 1) * NL < 64, "the wait counts to 63");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int of = wave % (S::WM * S::WN), quarter = wave / (S::WM * S::WN);
  const int wm = (of / S::WN) * 32 * MT, wn = (of % S::WN) * 32 * NT;
  LA ga;
  LW gw;
  ga.init(A, lda, m0, M, k0, wave, lane);
  gw.init(W, ldw, n0, N, k0, wave, lane);
  PtFrags<T, AK, S::rows> ra[MT];
  PtFrags<T, WK, S::cols> rw[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) ra[i].init(wm + 32 * i, lane);
#pragma unroll
  for (int j = 0; j < NT; ++j) rw[j].init(wn + 32 * j, lane);
  const int nk = (k1 - k0) / LA::KD;
  if (WK && w_end) {
    gw.end = (const char*)w_end + (size_t)n0 * sizeof(T);
    gw.at_end = nk - 1;
  }
  const uint32_t lds_at = (uint32_t)(uintptr_t)PT_LDS(lds);
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;
  auto load_all = [&](int slot, int stage) {
    const uint32_t at = lds_at + slot * S::stage;
#pragma unroll
    for (int n = 0; n < LA::L; ++n) ga.load_counted(at, stage, n, wave);
#pragma unroll
    for (int n = 0; n < LW::L; ++n) gw.load_counted(at + S::rows * 128, stage, n, wave);
  };
  // until at most `left` stages of this wave's loads are under way, its fragments read, and every wave here
  auto wait = [&](int left) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    auto upto = [&](auto n) {
      constexpr int v = decltype(n)::value * NL;
      __builtin_amdgcn_s_waitcnt(0x0070 | (v & 15) | ((v >> 4) << 14));
    };
    if (D > 3 && left >= 3) upto(std::integral_constant<int, (D > 3 ? 3 : 0)>{});
    else if (D > 2 && left == 2) upto(std::integral_constant<int, 2>{});
    else if (left == 1) upto(std::integral_constant<int, 1>{});
    else upto(std::integral_constant<int, 0>{});
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  pt_u32x4 fa[2][MT], fw[2][NT];
  auto frags = [&](int slot, int s, int buf) {
    const char* const la = lds + slot * S::stage;
#pragma unroll
    for (int n = 0; n < MT; ++n) fa[buf][n] = ra[n].read(la, s, lane);
#pragma unroll
    for (int n = 0; n < NT; ++n) fw[buf][n] = rw[n].read(la + S::rows * 128, s, lane);
  };
  auto mul = [&](int buf) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[j][i] = pt_mma(T(), fw[buf][j], fa[buf][i], acc[j][i]);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int u = 0; u < D - 1; ++u)
    if (u < nk) load_all(u, u);
  wait(min(D - 2, nk - 1));
  if constexpr (S::KW > 1) {
    frags(0, quarter, 0);
    for (int kt = 0, slot = 0; kt < nk; ++kt) {
      const int next = slot + 1 == D ? 0 : slot + 1, last = slot == 0 ? D - 1 : slot - 1;
      if (kt + D - 1 < nk) load_all(last, kt + D - 1);
      wait(max(0, min(D - 2, nk - 2 - kt)));
      frags(next, quarter, 1);
      mul(0);
#pragma unroll
      for (int n = 0; n < MT; ++n) fa[0][n] = fa[1][n];
#pragma unroll
      for (int n = 0; n < NT; ++n) fw[0][n] = fw[1][n];
      slot = next;
    }
    // (the others' sums, in the order of the quarters)
    auto each = [&](int q, auto f) {
      char* const at = lds + ((q - 1) * S::WM * S::WN + of) * MT * NT * 4096 + lane * 16;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) f(acc[j][i], 4 * x, (pt_f32x4*)(at + ((j * MT + i) * 4 + x) * 1024));
    };
    if (quarter)
      each(quarter, [](pt_f32x16& c, int e, pt_f32x4* to) { *to = pt_f32x4{c[e], c[e + 1], c[e + 2], c[e + 3]}; });
    __syncthreads();
    if (quarter) return;
#pragma unroll
    for (int q = 1; q < S::KW; ++q)
      each(q, [](pt_f32x16& c, int e, pt_f32x4* from) {
        const pt_f32x4 v = *from;
#pragma unroll
        for (int u = 0; u < 4; ++u) c[e + u] += v[u];
      });
    PT_WAVE_LDS_FENCE();
    return;
  }
  frags(0, 0, 0);
  for (int kt = 0, slot = 0; kt < nk; ++kt) {
    const int next = slot + 1 == D ? 0 : slot + 1, last = slot == 0 ? D - 1 : slot - 1;
    // the stage before this one is done with, for every wave: its place takes the one D - 1 ahead
    if (kt + D - 1 < nk) load_all(last, kt + D - 1);
    frags(slot, 1, 1);
    mul(0);
    frags(slot, 2, 0);
    mul(1);
    frags(slot, 3, 1);
    mul(0);
    // this wave's loads then under way: stages kt + 1 .. min(kt + D - 1, nk - 1), the first of which is wanted
    wait(max(0, min(D - 2, nk - 2 - kt)));
    frags(next, 0, 0);  // (after the last stage: of nothing)
    mul(1);
    slot = next;
  }
}

// The accumulators of a wave: element e of acc[j][i] is row 32 i + lane % 32, column 32 j + 8 (e / 4) + 4 (lane / 32) + e % 4.
__device__ __forceinline__ int pt_col(int j, int e, int hf) { return 32 * j + 8 * (e >> 2) + 4 * hf + (e & 3); }

// After the product a wave has 16 KB of it to itself: every wave has passed the last barrier with all that it read of the stages.
template <typename S>
__device__ __forceinline__ char* pt_wave_lds(char* la0, char* lw0, char* la1, char* lw1, int wave) {
  static_assert(S::rows == S::cols && S::rows * 512 == S::waves * 16384, "16 KB a wave");
  constexpr int per = S::waves / 4;
  char* const base = wave / per == 0 ? la0 : wave / per == 1 ? lw0 : wave / per == 2 ? la1 : lw1;
  return base + wave % per * 16384;
}

template <typename S>
__device__ __forceinline__ char* pt_any_wave_lds(char* ring, char* la0, char* lw0, char* la1, char* lw1) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if constexpr (S::RING > 2) return ring + wave * 16384;
  else return pt_wave_lds<S>(la0, lw0, la1, lw1, wave);
}

// One tile's product into acc, whichever way the shape keeps its stages (a ring's are one array), and the LDS a wave has afterwards.
#define PT_STAGES(S)                                                                   \
  constexpr bool kRing = S::RING > 2;                                                 \
  __shared__ __attribute__((aligned(16))) char ring[kRing ? S::RING * S::stage : 16]; \
  __shared__ __attribute__((aligned(16))) char la0[kRing ? 16 : S::rows * 128];       \
  __shared__ __attribute__((aligned(16))) char lw0[kRing ? 16 : S::cols * 128];       \
  __shared__ __attribute__((aligned(16))) char la1[kRing ? 16 : S::rows * 128];       \
  __shared__ __attribute__((aligned(16))) char lw1[kRing ? 16 : S::cols * 128];
#define PT_WAVE_LDS pt_any_wave_lds<S>(ring, la0, lw0, la1, lw1)
#define PT_PRODUCT(T, AK, WK, ...)                                            \
  if constexpr (kRing) pt_product_ring<T, AK, WK, S>(__VA_ARGS__, ring, acc); \
  else pt_product<T, AK, WK, S>(__VA_ARGS__, la0, lw0, la1, lw1, acc)

// The shapes in use.
using PtBig = PtShape<2, 4, 4, 2>;       // 256 x 256, 8 waves of 128 x 64, a CU to itself
using PtMid = PtShape<2, 2, 2, 2>;       // 128 x 128, 4 waves of 64 x 64, two blocks on a CU
using PtSmall = PtShape<2, 1, 1, 2, 4>;  // 64 x 64, 2 waves of 32 x 64, a ring of four stages, two blocks on a CU
using PtThin = PtShape<1, 1, 1, 2, 4, 4>;  // 32 x 64, 4 waves that each take a quarter of every stage, three blocks on a CU
template <typename S>
constexpr int pt_waves_eu = S::KW > 1 ? 3 : S::RING > 2 ? 1 : 2;  // for __launch_bounds__
template <typename S>
__device__ __forceinline__ bool pt_done(int wave) {  // after a product: this wave's results are another's
  return S::KW > 1 && wave >= S::WM * S::WN;
}

// Hands a wave's results out in memory order: 64 rows of its 64 columns at a time pass through its LDS as float (16-byte chunks XORed with
// the row), since a store from the accumulators would touch 32 rows with 16 bytes each.  sink(row, col, v, it): N (4 or 8)
// consecutive columns of a row, sixteen or eight lanes a row, the pass's it-th call; before(pass): called before a pass's 64 rows.
// (32 rows where a wave has no more)
template <int N, int MT, typename B, typename O>
__device__ __forceinline__ void pt_hand_out(char* ep, int lane, const pt_f32x16 (&acc)[2][MT], B before, O sink) {
  constexpr int PR = MT > 1 ? 64 : 32, IP = PR / 32;
  static_assert(MT % IP == 0 && (N == 4 || N == 8), "whole passes");
  const int l32 = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int pass = 0; pass < MT / IP; ++pass) {
    before(pass);
#pragma unroll
    for (int i = 0; i < IP; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const pt_f32x16& a = acc[j][IP * pass + i];
          const pt_f32x4 v = {a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
          *(pt_f32x4*)(ep + (32 * i + l32) * 256 + (((8 * j + 2 * q + hf) ^ (l32 & 15)) << 4)) = v;
        }
    PT_WAVE_LDS_FENCE();
    constexpr int LR = 64 / N, RI = 64 / LR;  // lanes of a row, rows of an instruction
    const int rd_row = lane / LR, rd_c = lane % LR;
#pragma unroll
    for (int it = 0; it < PR / RI; ++it) {
      const int row = RI * it + rd_row;
      if constexpr (N == 4) {
        sink(PR * pass + row, rd_c * 4, *(const pt_f32x4*)(ep + row * 256 + ((rd_c ^ (row & 15)) << 4)), it);
      } else {
        float v[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const pt_f32x4 x = *(const pt_f32x4*)(ep + row * 256 + (((2 * rd_c + k) ^ (row & 15)) << 4));
#pragma unroll
          for (int u = 0; u < 4; ++u) v[4 * k + u] = x[u];
        }
        sink(PR * pass + row, rd_c * 8, v, it);
      }
    }
    PT_WAVE_LDS_FENCE();
  }
}
struct PtNothing {
  __device__ void operator()(int) const {}
};

// The transpose of a wave's results as half: sink(col, row, v) gets eight consecutive rows of a column.  32 MT rows of 128 bytes in LDS,
// read through the transposing LDS read (see PtFrags).
template <int MT, typename O>
__device__ __forceinline__ void pt_hand_out_transposed(char* ep, int lane, const pt_f32x16 (&acc)[2][MT], O sink) {
  typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
  typedef __attribute__((ext_vector_type(4))) short s16x4;
  typedef __attribute__((address_space(3))) s16x4* lds4;
  const int l32 = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f16x4 h;
#pragma unroll
        for (int u = 0; u < 4; ++u) h[u] = (half_t)acc[j][i][4 * q + u];
        *(f16x4*)(ep + (32 * i + l32) * 128 + (((4 * j + q) ^ (l32 & 7)) << 4) + 8 * hf) = h;
      }
  PT_WAVE_LDS_FENCE();
  const int r = lane & 15, oct = lane >> 4;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int c0 = 0; c0 < 64; c0 += 16) {
      pt_u32x4 v;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = 32 * i + 8 * oct + 4 * k + (r >> 2), chunk = ((c0 >> 3) + ((r & 3) >> 1)) ^ (row & 7);
        const pt_u32x2 x = __builtin_bit_cast(
            pt_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(ep + row * 128 + chunk * 16 + (r & 1) * 8)));
        v[2 * k] = x[0];
        v[2 * k + 1] = x[1];
      }
      sink(c0 + r, 32 * i + 8 * oct, v);
    }
  PT_WAVE_LDS_FENCE();
}

__device__ __forceinline__ uint16_t pt_bits(half_t, float v) { return __builtin_bit_cast(uint16_t, (half_t)v); }
__device__ __forceinline__ uint16_t pt_bits(bfloat, float v) { return __builtin_bit_cast(uint16_t, (bfloat)v); }
template <typename T>
__device__ __forceinline__ pt_u32x4 pt_pack8(const float (&v)[8]) {
  pt_u32x4 r;
#pragma unroll
  for (int u = 0; u < 4; ++u) r[u] = (uint32_t)pt_bits(T(), v[2 * u]) | (uint32_t)pt_bits(T(), v[2 * u + 1]) << 16;
  return r;
}

// Tile t of nb_m x nb_n: consecutive tiles walk four row tiles for each column tile.
__device__ __forceinline__ void pt_tile_pos(int t, int nb_m, int nb_n, int& tm, int& tn) {
  constexpr int G = 4;
  const int grp = t / (G * nb_n), r = t - grp * G * nb_n, gm = min(G, nb_m - grp * G);
  tm = grp * G + r % gm;
  tn = r / gm;
}
// Tile t of the lower triangle (tm >= tn) of a square of tiles.
__device__ __forceinline__ void pt_tile_triangle(int t, int& tm, int& tn) {
  tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
  while (tm * (tm + 1) / 2 > t) --tm;
  tn = t - tm * (tm + 1) / 2;
}
// Work item of this block of a launch of `items` (grid: pt_grid); -1: none.  Block b runs on XCD b % 8.
// An XCD takes a contiguous run of items, whose operands its L2 then holds.
__device__ __forceinline__ int pt_item(int items) {
  const int per = (items + 7) >> 3, b = (int)blockIdx.x, it = (b & 7) * per + (b >> 3);
  return (b >> 3) < per && it < items ? it : -1;
}
// Or the XCDs go through the items together, 256 neighbours at a time, 32 in a row to each: for sums over a long K, whose operands the
// XCDs then share in the last cache (13,568 rows, 50,304 x 2,560: dh 2.96 -> 2.83 ms, dW 2.82 -> 2.66; the products over K = 2,560 of
// the same call 3.13 -> 3.25 the other way).
__device__ __forceinline__ int pt_item_rounds(int items) {
  const int b = (int)blockIdx.x, x = b & 7, r = b >> 3, full = items / 256 * 32;
  if (r < full) return (r >> 5) * 256 + x * 32 + (r & 31);
  const int rem = items % 256, per = (rem + 7) >> 3, it = items - rem + x * per + (r - full);
  return r - full < per && it < items ? it : -1;
}
inline unsigned pt_grid(int items) { return 8u * (unsigned)((items + 7) / 8); }

}  // namespace rlhf
