// Orthogonalised updates.  A matrix G is brought towards the orthogonal factor of its singular value decomposition by the quintic
// Newton-Schulz iteration: X = G / (|G|_F + eps), then `steps` times
//   A = X X^T,  B = b A + c A^2,  X <- a X + B X      (a, b, c = 3.4445, -4.7750, 2.0315)
// which maps each singular value s to a s + b s^3 + c s^5 and brings those of 0.0015 and more to 0.68 .. 1.21 in five.  A matrix
// with more rows than columns is taken from the other side, A = X^T X and X <- a X + X B, in its own layout: which side of a
// product an operand stands on is a matter of reading it row-major or K-major.
//
// Precision.  The products run on fp16 operands with fp32 sums.  The iteration enlarges what lies along small singular
// values up to a^5 = 485 times, rounding errors of X included: with X itself in fp16 a gradient of few strong directions
// over weak noise comes out 1 to 3 % off, in bfloat16 9 to 18 %.  So X is kept as two fp16 halves (22 bits) and only the
// operands of the products are rounded: 0.02 to 0.2 % over all spectra tried.  X is scaled by 2^11 and A and B by 2^12, which puts
// entries down to the sizes that matter into fp16's normal range and leaves the largest (singular values stay below 1.21) a
// factor of ten below its end.  The norm is summed in double.
//
// A and B are symmetric: the tiles of the lower triangle are multiplied and stored twice.  Matrices lie in the workspace padded
// with zeros to multiples of 64, which the iteration keeps zero.  All matrices of a call share its launches.
//
// What bounds it.  Large layers (eight matrices, two layers of width 2,560: 8.1 ms): the products, 3.1 s^2 l + 1.1 s^3 operations a step and matrix
// of s x l (s <= l), 960 TFLOP/s over the five steps, and 8 bytes an element a step for X's halves, which the update's tiles read and
// write at their ends, when their CUs' matrix cores wait; the first two passes, 0.69 ms, move their bytes at 4.7 TB/s and more.
// Few or small matrices: 15 launches of tiles that depend on each other, 6 to 10 us each (1,025 x 333: 132 us, 17 launches and the norm).
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstring>

#include "common.h"
#include "muon.h"
#include "product_tile.h"

namespace rlhf {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kXScale = 2048.f, kAScale = 4096.f;
constexpr int kProbs = kMuonGroup;  // of a launch
constexpr int kNormElems = 4096;  // elements of a block of the norm
constexpr size_t kGroupElems = (size_t)1 << 28;

struct Prob {
  half_t *xh[2], *xl[2];  // [rp][ld], the high and the low half, of this step and the next
  half_t *a, *b;          // [sp][sp]
  double* part;           // the norm's partial sums
  float* scale;           // kXScale / (norm + eps)
  MuonMatrix m;
  int rp, ld, sp;         // rows, columns, and the shorter of them, padded
  float step;             // lr rms sqrt(max(rows, cols))
  int vec;                // 16-byte accesses to the caller's arrays: eight elements of a row start where they may
};
enum Part { kNorm, kSplit, kGram, kPoly, kUpdate, kParts };
// What the launches of a group share.  It lies in the workspace, put there before them: as an argument of each, it would be fetched
// from the argument segment, line after line, by every block.
struct Group {
  MuonScalars c;
  int count;
  uint32_t items[kParts];         // all work items
  uint32_t first[kParts][kProbs]; // first work item of each problem, ~0 beyond the last
  uint32_t start[kParts][9];      // tiles that are dealt in runs: where each XCD's begins; split[]: every problem is dealt to all XCDs
  uint32_t split[kParts];         // (items are then eighths of them)
  Prob p[kProbs];
};
static_assert(kProbs < 64, "a problem is found by the lanes of a wave");

struct Words {
  uint32_t w[960];
};
__global__ void __launch_bounds__(256) muon_table_kernel(Words in, int n, uint32_t* out) {
  for (int i = threadIdx.x; i < n; i += 256) out[i] = in.w[i];
}

// The problem of a work item of `part`, the item's index within it, and how many it has.
__device__ __forceinline__ const Prob& find_prob(const Group* __restrict__ g, Part part, uint32_t item, int& index, int& of) {
  const int lane = threadIdx.x & 63;
  const uint32_t first = lane < kProbs ? g->first[part][lane] : ~0u;
  const int at = __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= item)) - 1);  // (first[0] is 0)
  const uint32_t from = (uint32_t)__builtin_amdgcn_readlane((int)first, at), to = (uint32_t)__builtin_amdgcn_readlane((int)first, at + 1);
  index = (int)(item - from);
  of = (int)(min(to, g->items[part]) - from);
  return g->p[at];
}
// Tiles: block b runs on XCD b % 8.  Few problems of many tiles: every XCD takes an eighth of each, a run of neighbours, and all work
// on a problem at a time, whose operands then are in the last cache.  Many of few tiles: an XCD takes a run of neighbouring tiles of as
// much work as the others', so that a problem's operands go to one XCD or two (24 matrices of width 512: A^2 21 -> 13 us a launch;
// eight of the 2.8B layers the other way round 5 % slower).  -1: none.
__device__ __forceinline__ const Prob& find_tile(const Group* __restrict__ g, Part part, int& tile) {
  const uint32_t x = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const bool split = g->split[part] != 0;
  const uint32_t item = split ? slot : g->start[part][x] + slot;
  const bool none = !split && item >= g->start[part][x + 1];
  int index, of;
  const Prob& p = find_prob(g, part, min(item, g->items[part] - 1), index, of);
  tile = __builtin_amdgcn_readfirstlane(none ? -1 : split ? (int)x * of + index : index);
  return p;
}

__device__ __forceinline__ float bf16_at(const void* p, size_t i) { return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16); }

// v as two halves.  The value and its high half are kept opaque: a multiplication before the first rounding would be fused into it
// for one of its uses and not for the other, and where the two roundings part, h and l would belong to different numbers, a whole
// unit of h apart.
__device__ __forceinline__ void split_halves(float v, half_t& h, half_t& l) {
  asm volatile("" : "+v"(v));
  float back = (float)(half_t)v;
  asm volatile("" : "+v"(back));
  h = (half_t)back;
  l = (half_t)(v - back);
}

// What is orthogonalised at element i, from the updated momentum.
__device__ __forceinline__ float source_at(const Prob& p, const MuonScalars& c, size_t i) {
  if (p.m.src) return c.src_bf16 ? bf16_at(p.m.src, i) : ((const float*)p.m.src)[i];
  const float v = p.m.moment[i];
  return c.nesterov ? c.omb * (c.grad_scale * p.m.grad[i]) + c.beta * v : v;
}

// The same of eight neighbours, all arrays 16-byte aligned there.
__device__ __forceinline__ void source8(const Prob& p, const MuonScalars& c, size_t i, float (&v)[8]) {
  if (p.m.src && c.src_bf16) {
    const pt_u32x4 r = *(const pt_u32x4*)((const uint16_t*)p.m.src + i);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v[2 * u] = __uint_as_float(r[u] << 16);
      v[2 * u + 1] = __uint_as_float(r[u] & 0xFFFF0000u);
    }
    return;
  }
  const float* const src = p.m.src ? (const float*)p.m.src : p.m.moment;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const pt_f32x4 m = *(const pt_f32x4*)(src + i + 4 * k);
    pt_f32x4 gr = {0.f, 0.f, 0.f, 0.f};
    if (!p.m.src && c.nesterov) gr = *(const pt_f32x4*)(p.m.grad + i + 4 * k);
#pragma unroll
    for (int u = 0; u < 4; ++u) v[4 * k + u] = !p.m.src && c.nesterov ? c.omb * (c.grad_scale * gr[u]) + c.beta * m[u] : m[u];
  }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
  auto step = [&](auto o) {
    constexpr int O = decltype(o)::value;
    v += __hiloint2double(lane_xor<O>(__double2hiint(v)), lane_xor<O>(__double2loint(v)));
  };
  step(std::integral_constant<int, 32>{});
  step(std::integral_constant<int, 16>{});
  step(std::integral_constant<int, 8>{});
  step(std::integral_constant<int, 4>{});
  step(std::integral_constant<int, 2>{});
  step(std::integral_constant<int, 1>{});
  return v;
}

// The momentum's update, and the sum of squares of 4,096 elements.  Bound by its bytes, 12 an element (157 M elements: 0.35 ms, 5.4 TB/s).
// Blocks of 16,384 elements were no faster there, and slower where there are few (1,025 x 333: 13.6 us, so 5.5).
__global__ void __launch_bounds__(256) muon_norm_kernel(const Group* __restrict__ g) {
  const MuonScalars c = g->c;
  __shared__ double sh[4];
  int block, of;
  const Prob& p = find_prob(g, kNorm, blockIdx.x, block, of);
  const size_t n = (size_t)p.m.rows * p.m.cols, i0 = (size_t)block * kNormElems, i1 = min(n, i0 + kNormElems);
  double sum = 0.0;
  if (p.vec) {  // (i1 - i0 is a multiple of eight)
    for (size_t i = i0 + 8 * threadIdx.x; i < i1; i += 2048) {
      float v[8];
      if (!p.m.src) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          pt_f32x4 m = *(const pt_f32x4*)(p.m.moment + i + 4 * k);
          const pt_f32x4 gr = *(const pt_f32x4*)(p.m.grad + i + 4 * k);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            m[u] = c.beta * m[u] + c.omb * (c.grad_scale * gr[u]);
            v[4 * k + u] = c.nesterov ? c.omb * (c.grad_scale * gr[u]) + c.beta * m[u] : m[u];
          }
          *(pt_f32x4*)(p.m.moment + i + 4 * k) = m;
        }
      } else {
        source8(p, c, i, v);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) sum += (double)v[u] * (double)v[u];
    }
  }
  for (size_t i = p.vec ? i1 : i0 + threadIdx.x; i < i1; i += 256) {
    if (!p.m.src) p.m.moment[i] = c.beta * p.m.moment[i] + c.omb * (c.grad_scale * p.m.grad[i]);
    const double v = source_at(p, c, i);
    sum += v * v;
  }
  sum = wave_sum_f64(sum);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.part[block] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__global__ void __launch_bounds__(256) muon_scale_kernel(const Group* __restrict__ g) {
  const MuonScalars c = g->c;
  __shared__ double sh[256];
  const Prob& p = g->p[blockIdx.x];
  const int blocks = (int)(((size_t)p.m.rows * p.m.cols + kNormElems - 1) / kNormElems);
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) sum += p.part[i];
  sh[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 128; o; o /= 2) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double norm = sqrt(sh[0]) + c.eps;
    *p.scale = norm != norm ? NAN : (float)fmin((double)kXScale / norm, 3e38);  // (finite, so that nothing stays 0)
  }
}

// X = scale * source as two halves, zero in the padding; eight columns a thread.  Bound by its bytes, 12 an element with nesterov
// (157 M elements: 0.34 ms, 5.6 TB/s).
__global__ void __launch_bounds__(256) muon_split_kernel(const Group* __restrict__ g) {
  const MuonScalars c = g->c;
  int block, of;
  const Prob& p = find_prob(g, kSplit, blockIdx.x, block, of);
  const uint32_t chunk = (uint32_t)block * 256 + threadIdx.x, per_row = (uint32_t)p.ld / 8;
  const uint32_t row = chunk / per_row, col = (chunk - row * per_row) * 8;
  if (row >= (uint32_t)p.rp) return;
  const float s = *p.scale;
  typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
  f16x8 h, l;
  float v[8];
  const size_t at = (size_t)row * p.m.cols + col;
  if (p.vec && row < (uint32_t)p.m.rows && col + 8 <= (uint32_t)p.m.cols) {
    source8(p, c, at, v);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = row < (uint32_t)p.m.rows && col + u < (uint32_t)p.m.cols ? source_at(p, c, at + u) : 0.f;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    half_t hu, lu;
    split_halves(s * v[u], hu, lu);
    h[u] = hu;
    l[u] = lu;
  }
  *(f16x8*)(p.xh[0] + (size_t)row * p.ld + col) = h;
  *(f16x8*)(p.xl[0] + (size_t)row * p.ld + col) = l;
}

// A symmetric tile: alpha * acc + (IN) beta * in, stored at its place and, off the diagonal, mirrored.
template <typename S, bool IN>
__device__ __forceinline__ void store_symmetric(pt_f32x16 (&acc)[S::NT][S::MT], const half_t* in, half_t* out, int ld, int tm, int tn,
                                                float alpha, float beta, char* ep) {
  constexpr int MT = S::MT;
  typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hf = lane >> 5;
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
  if (row0 >= ld || col0 >= ld) return;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = min(row0 + 32 * i + l32, ld - 1);
    f16x4 x[2][4];
    if (IN) {  // (a wave's 64 columns exist or do not as a whole)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) x[j][q] = *(const f16x4*)(in + (size_t)row * ld + col0 + pt_col(j, 4 * q, hf));
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float v = alpha * acc[j][i][e];
        if (IN) v += beta * (float)x[j][e >> 2][e & 3];
        acc[j][i][e] = v;
      }
  }
  if (tm != tn)
    pt_hand_out_transposed<MT>(ep, lane, acc, [&](int c, int r, pt_u32x4 v) {
      if (row0 + r < ld) *(pt_u32x4*)(out + (size_t)(col0 + c) * ld + row0 + r) = v;
    });
  pt_hand_out<8, MT>(ep, lane, acc, PtNothing(), [&](int r, int c, const float(&v)[8], int) {
    if (row0 + r < ld) *(pt_u32x4*)(out + (size_t)(row0 + r) * ld + col0 + c) = pt_pack8<half_t>(v);
  });
}

// A = X X^T (the shorter side's), scaled.  (Eight matrices of two layers of width 2,560, l = 2,560 to 10,240: 0.45 ms a step; 16 of 2,048 x 2,048
// 0.19 ms.)
template <typename S>
__global__ void __launch_bounds__(64 * S::waves, pt_waves_eu<S>) muon_gram_kernel(const Group* __restrict__ g, int cur) {
  PT_STAGES(S)
  int tile;
  const Prob& p = find_tile(g, kGram, tile);
  if (tile < 0) return;
  int tm, tn;
  pt_tile_triangle(tile, tm, tn);
  if (tm * S::rows >= p.sp) return;
  pt_f32x16 acc[S::NT][S::MT];
  const half_t* const x = p.xh[cur];
  if (p.m.rows > p.m.cols)
    PT_PRODUCT(half_t, true, true, x, p.ld, tm * S::rows, p.sp, x, p.ld, tn * S::cols, p.sp, 0, p.rp, nullptr);
  else
    PT_PRODUCT(half_t, false, false, x, p.ld, tm * S::rows, p.sp, x, p.ld, tn * S::cols, p.sp, 0, p.ld, nullptr);
  store_symmetric<S, false>(acc, nullptr, p.a, p.sp, tm, tn, kAScale / (kXScale * kXScale), 0.f, PT_WAVE_LDS);
}

// B = b A + c A^2 (0.17 and 0.21 ms)
template <typename S>
__global__ void __launch_bounds__(64 * S::waves, pt_waves_eu<S>) muon_poly_kernel(const Group* __restrict__ g) {
  PT_STAGES(S)
  int tile;
  const Prob& p = find_tile(g, kPoly, tile);
  if (tile < 0) return;
  int tm, tn;
  pt_tile_triangle(tile, tm, tn);
  if (tm * S::rows >= p.sp) return;
  pt_f32x16 acc[S::NT][S::MT];
  PT_PRODUCT(half_t, false, false, p.a, p.sp, tm * S::rows, p.sp, p.a, p.sp, tn * S::cols, p.sp, 0, p.sp, nullptr);
  store_symmetric<S, true>(acc, p.a, p.b, p.sp, tm, tn, kC / kAScale, kB, PT_WAVE_LDS);
}

// X <- a X + B X, or after the last step what becomes of it.  (0.83 and 0.32 ms: the product, and 8 bytes an element.  Stores that
// bypass the caches, requests of X halfway through the product and tiles that start apart from each other all gained nothing.)
template <typename S>
__global__ void __launch_bounds__(64 * S::waves, pt_waves_eu<S>) muon_update_kernel(const Group* __restrict__ g, int cur, int last) {
  const MuonScalars c = g->c;
  PT_STAGES(S)
  constexpr int MT = S::MT;
  int tile;
  const Prob& p = find_tile(g, kUpdate, tile);
  const int nb_m = (p.rp + S::rows - 1) / S::rows, nb_n = (p.ld + S::cols - 1) / S::cols;
  if (tile < 0 || tile >= nb_m * nb_n) return;
  int tm, tn;
  pt_tile_pos(tile, nb_m, nb_n, tm, tn);
  pt_f32x16 acc[2][MT];
  if (p.m.rows > p.m.cols)
    PT_PRODUCT(half_t, false, false, p.xh[cur], p.ld, tm * S::rows, p.rp, p.b, p.sp, tn * S::cols, p.sp, 0, p.sp, nullptr);
  else
    PT_PRODUCT(half_t, false, true, p.b, p.sp, tm * S::rows, p.sp, p.xh[cur], p.ld, tn * S::cols, p.ld, 0, p.sp, nullptr);
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
  if (row0 >= p.rp || col0 >= p.ld) return;
  typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
  const int rows = p.m.rows, cols = p.m.cols, rd_row = lane >> 3, rd_c = lane & 7;
  const half_t* const xh = p.xh[cur] + (size_t)row0 * p.ld + col0;
  const half_t* const xl = p.xl[cur] + (size_t)row0 * p.ld + col0;
  half_t* const nh = p.xh[cur ^ 1] + (size_t)row0 * p.ld + col0;
  half_t* const nl = p.xl[cur ^ 1] + (size_t)row0 * p.ld + col0;
  f16x8 h[MT > 1 ? 8 : 4], l[MT > 1 ? 8 : 4];  // this pass's X, requested before the results go through LDS
  constexpr int PR = MT > 1 ? 64 : 32, NI = PR / 8;
  pt_hand_out<8, MT>(
      PT_WAVE_LDS, lane, acc,
      [&](int pass) {
#pragma unroll
        for (int it = 0; it < NI; ++it) {
          const size_t i = (size_t)min(PR * pass + 8 * it + rd_row, p.rp - 1 - row0) * p.ld + 8 * rd_c;
          h[it] = *(const f16x8*)(xh + i);
          l[it] = *(const f16x8*)(xl + i);
        }
      },
      [&](int r, int cc, float(&v)[8], int it) {
        const int row = row0 + r, col = col0 + cc;
        if (row >= p.rp) return;
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = fmaf(v[u], 1.f / kAScale, kA * ((float)h[it][u] + (float)l[it][u]));
        if (!last) {
          f16x8 a, b;
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            half_t hu, lu;
            split_halves(v[u], hu, lu);
            a[u] = hu;
            b[u] = lu;
          }
          const size_t i = (size_t)r * p.ld + cc;
          *(f16x8*)(nh + i) = a;
          *(f16x8*)(nl + i) = b;
          return;
        }
        if (row >= rows) return;
        const size_t o = (size_t)row * cols + col;
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] *= 1.f / kXScale;
        if (p.vec && col + 8 <= cols) {
          if (!p.m.src) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              pt_f32x4 w = *(const pt_f32x4*)(p.m.param + o + 4 * k);
#pragma unroll
              for (int u = 0; u < 4; ++u) v[4 * k + u] = w[u] = c.decay * w[u] - p.step * v[4 * k + u];
              *(pt_f32x4*)(p.m.param + o + 4 * k) = w;
            }
          }
          uint16_t* const to = p.m.src ? p.m.out : p.m.param_bf16;
          if (to) *(pt_u32x4*)(to + o) = pt_pack8<bfloat>(v);
          return;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if (col + u >= cols) break;
          if (p.m.src) {
            p.m.out[o + u] = pt_bits(bfloat(), v[u]);
          } else {
            const float w = c.decay * p.m.param[o + u] - p.step * v[u];
            p.m.param[o + u] = w;
            if (p.m.param_bf16) p.m.param_bf16[o + u] = pt_bits(bfloat(), w);
          }
        }
      });
}

int pad64(int n) { return (n + 63) & ~63; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
int norm_blocks(int rows, int cols) { return (int)(((size_t)rows * cols + kNormElems - 1) / kNormElems); }

// The matrices from `from` on that go together: up to 2^28 elements (but one at least).
int group_end(const MuonMatrix* ms, int from, int count) {
  size_t n = 0;
  int i = from;
  for (; i < count; ++i) {
    n += (size_t)pad64(ms[i].rows) * pad64(ms[i].cols);
    if (i > from && n > kGroupElems) break;
  }
  return i;
}

// Lays the group's buffers into the workspace from `base` on (null: measures); returns the end.
size_t lay_out(Group* g, char* base, const MuonMatrix* ms, int from, int to) {
  size_t off = align256(sizeof(Group));  // (the table's place)
  auto take = [&](size_t bytes) {
    char* const at = base ? base + off : nullptr;
    off += align256(bytes);
    return at;
  };
  for (int i = from; i < to; ++i) {
    const int rp = pad64(ms[i].rows), ld = pad64(ms[i].cols), sp = std::min(rp, ld);
    Prob dummy;
    Prob& p = g ? g->p[i - from] : dummy;
    for (int k = 0; k < 2; ++k) {
      p.xh[k] = (half_t*)take((size_t)rp * ld * 2);
      p.xl[k] = (half_t*)take((size_t)rp * ld * 2);
    }
    p.a = (half_t*)take((size_t)sp * sp * 2);
    p.b = (half_t*)take((size_t)sp * sp * 2);
    p.part = (double*)take((size_t)norm_blocks(ms[i].rows, ms[i].cols) * 8);
    p.scale = (float*)take(4);
    p.rp = rp;
    p.ld = ld;
    p.sp = sp;
  }
  return off;
}

template <typename F>
void number(Group& g, Part part, F items) {
  uint32_t n = 0;
  for (int i = 0; i < kProbs; ++i) {
    g.first[part][i] = i < g.count ? n : ~0u;
    if (i < g.count) n += (uint32_t)items(g.p[i]);
  }
  g.items[part] = n;
}
int up(int n, int t) { return (n + t - 1) / t; }
int triangle(int n) { return n * (n + 1) / 2; }

// What runs on tiles: the number of them and the length of their sums.
struct Tiles {
  int (*count)(const Prob&, int tile);
  int (*depth)(const Prob&);
};
const Tiles kGramTiles = {[](const Prob& p, int t) { return triangle(up(p.sp, t)); }, [](const Prob& p) { return std::max(p.rp, p.ld); }};
const Tiles kPolyTiles = {[](const Prob& p, int t) { return triangle(up(p.sp, t)); }, [](const Prob& p) { return p.sp; }};
const Tiles kUpdateTiles = {[](const Prob& p, int t) { return up(p.rp, t) * up(p.ld, t); }, [](const Prob& p) { return p.sp; }};

// Time of a launch's rounds of tiles: `slots` places, `stage` us a stage and `more` stages' worth for a tile's start and end.
double rounds_us(const Group& g, const Tiles& t, int tile, int slots, double stage, double more) {
  double work = 0, most = 0;
  for (int i = 0; i < g.count; ++i) {
    work += (double)t.count(g.p[i], tile) * t.depth(g.p[i]);
    most = std::max(most, (double)t.depth(g.p[i]));
  }
  return std::ceil(work / most / slots) * (most / 64 + more) * stage;
}

enum Shape { kBig, kMid, kSmall };
constexpr int kTile[] = {256, 128, 64}, kThreads[] = {512, 256, 128};

// The tiles of a launch.  Up to half as many middle ones as there are CUs leave most of the chip idle and wait for their loads: small
// ones, four times as many, with three stages under way (one matrix of 768 x 768 225 -> 149 us, of 333 x 1025 213 -> 138, the four of a
// layer of width 768 410 -> 337; 24 of the 70M shape 616 -> 719 the other way).  Else a large tile takes 1.95 us a stage and two
// middle ones on a CU, half of its products, 1.5.
Shape shape_of(const Group& g, const Tiles& t) {
  int mids = 0;
  for (int i = 0; i < g.count; ++i) mids += t.count(g.p[i], kTile[kMid]);
  if (mids <= 128) return kSmall;
  return rounds_us(g, t, kTile[kBig], 256, 1.95, 8) <= rounds_us(g, t, kTile[kMid], 512, 1.5, 5) ? kBig : kMid;
}

Shape number_tiles(Group& g, Part part, const Tiles& t) {
  const Shape c = shape_of(g, t);
  double work = 0;
  int tiles = 0;
  for (int i = 0; i < g.count; ++i) {
    work += (double)t.count(g.p[i], kTile[c]) * t.depth(g.p[i]);
    tiles += t.count(g.p[i], kTile[c]);
  }
  g.split[part] = tiles >= 32 * g.count;
  if (g.split[part]) {
    number(g, part, [&](const Prob& p) { return up(t.count(p, kTile[c]), 8); });
    return c;
  }
  number(g, part, [&](const Prob& p) { return t.count(p, kTile[c]); });
  double done = 0;
  int x = 0;
  for (int i = 0; i < g.count; ++i) {
    const double each = t.depth(g.p[i]), end = done + each * t.count(g.p[i], kTile[c]);
    for (; x < 8 && work * x / 8 < end; ++x) g.start[part][x] = g.first[part][i] + (uint32_t)((work * x / 8 - done) / each);
    done = end;
  }
  for (; x < 9; ++x) g.start[part][x] = g.items[part];
  return c;
}
template <typename K, typename... A>
void on_tiles(const Group& g, const Group* dev, Part part, Shape c, hipStream_t s, K big, K mid, K small, A... args) {
  uint32_t most = g.split[part] ? g.items[part] : 0;
  for (int x = 0; x < 8 && !g.split[part]; ++x) most = std::max(most, g.start[part][x + 1] - g.start[part][x]);
  hipLaunchKernelGGL(c == kBig ? big : c == kMid ? mid : small, dim3(8 * most), dim3(kThreads[c]), 0, s, dev, args...);
}

}  // namespace

size_t muon_workspace_bytes(const MuonMatrix* ms, int count) {
  size_t most = 0;
  for (int from = 0; from < count;) {
    const int to = group_end(ms, from, count);
    most = std::max(most, lay_out(nullptr, nullptr, ms, from, to));
    from = to;
  }
  return most;
}

hipError_t launch_muon(const MuonMatrix* ms, int count, const MuonScalars& c, void* workspace, hipStream_t s) {
  for (int from = 0; from < count;) {
    const int to = group_end(ms, from, count);
    Group g;
    g.count = to - from;
    g.c = c;
    lay_out(&g, (char*)workspace, ms, from, to);
    for (int i = 0; i < g.count; ++i) {
      const MuonMatrix& m = g.p[i].m = ms[from + i];
      g.p[i].step = (float)(c.lr_rms * std::sqrt((double)std::max(m.rows, m.cols)));
      const uintptr_t bases = (uintptr_t)m.src | (uintptr_t)m.out | (uintptr_t)m.param | (uintptr_t)m.grad | (uintptr_t)m.moment |
                              (uintptr_t)m.param_bf16;
      g.p[i].vec = m.cols % 8 == 0 && (bases & 15) == 0;
    }
    std::sort(g.p, g.p + g.count, [](const Prob& a, const Prob& b) { return std::max(a.rp, a.ld) > std::max(b.rp, b.ld); });
    number(g, kNorm, [](const Prob& p) { return norm_blocks(p.m.rows, p.m.cols); });
    number(g, kSplit, [](const Prob& p) { return (int)(((size_t)p.rp * p.ld / 8 + 255) / 256); });
    const Shape gram = number_tiles(g, kGram, kGramTiles), poly = number_tiles(g, kPoly, kPolyTiles), update = number_tiles(g, kUpdate, kUpdateTiles);
    Group* const dev = (Group*)workspace;
    const size_t words = (offsetof(Group, p) + g.count * sizeof(Prob)) / 4;
    for (size_t at = 0; at < words; at += sizeof(Words) / 4) {
      const int n = (int)std::min(words - at, sizeof(Words) / 4);
      Words w;
      std::memcpy(w.w, (const uint32_t*)&g + at, (size_t)n * 4);
      hipLaunchKernelGGL(muon_table_kernel, dim3(1), dim3(256), 0, s, w, n, (uint32_t*)dev + at);
    }
    hipLaunchKernelGGL(muon_norm_kernel, dim3(g.items[kNorm]), dim3(256), 0, s, dev);
    hipLaunchKernelGGL(muon_scale_kernel, dim3(g.count), dim3(256), 0, s, dev);
    hipLaunchKernelGGL(muon_split_kernel, dim3(g.items[kSplit]), dim3(256), 0, s, dev);
    for (int k = 0; k < c.steps; ++k) {
      const int cur = k & 1;
      on_tiles(g, dev, kGram, gram, s, muon_gram_kernel<PtBig>, muon_gram_kernel<PtMid>, muon_gram_kernel<PtSmall>, cur);
      on_tiles(g, dev, kPoly, poly, s, muon_poly_kernel<PtBig>, muon_poly_kernel<PtMid>, muon_poly_kernel<PtSmall>);
      on_tiles(g, dev, kUpdate, update, s, muon_update_kernel<PtBig>, muon_update_kernel<PtMid>, muon_update_kernel<PtSmall>, cur,
               (int)(k + 1 == c.steps));
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    from = to;
  }
  return hipSuccess;
}

}  // namespace rlhf
