// Orthogonalised updates.  A matrix G is brought towards the orthogonal factor of its singular value decomposition by the quintic
// Newton-Schulz iteration: X = G / (|G|_F + eps), then `steps` times
//   A = X X^T,  B = b A + c A^2,  X <- a X + B X      (a, b, c = 3.4445, -4.7750, 2.0315)
// which maps each singular value s to a s + b s^3 + c s^5 and brings those of 1e-3 and more near 1 in five steps.  A matrix
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
#include <algorithm>
#include <cmath>

#include "common.h"
#include "muon.h"
#include "product_tile.h"

namespace rlhf {

namespace {

using PtBig = PtShape<2, 4, 4, 2>;
using PtMid = PtShape<2, 2, 2, 2>;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kXScale = 2048.f, kAScale = 4096.f;
constexpr int kProbs = kMuonGroup;
constexpr int kNormElems = 16384;  // elements of a block of the norm
constexpr size_t kGroupElems = (size_t)1 << 28;

struct Prob {
  half_t *xh[2], *xl[2];  // [rp][ld], the high and the low half, of this step and the next
  half_t *a, *b;          // [sp][sp]
  double* part;           // the norm's partial sums
  float* scale;           // kXScale / (norm + eps)
  MuonMatrix m;
  int rp, ld, sp;         // rows, columns, and the shorter of them, padded
  float step;             // lr rms sqrt(max(rows, cols))
};
struct Group {
  Prob p[kProbs];
  uint32_t first[kProbs];  // first work item of each
  int count;
  uint32_t items;
  MuonScalars c;
};

__device__ __forceinline__ int find_prob(const Group& g, uint32_t item) {
  int at = 0;
  for (int i = 1; i < g.count; ++i)
    if (g.first[i] <= item) at = i;
  return at;
}

__device__ __forceinline__ float bf16_at(const void* p, size_t i) { return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16); }

// What is orthogonalised at element i, from the updated momentum.
__device__ __forceinline__ float source_at(const Prob& p, const MuonScalars& c, size_t i) {
  if (p.m.src) return c.src_bf16 ? bf16_at(p.m.src, i) : ((const float*)p.m.src)[i];
  const float v = p.m.moment[i];
  return c.nesterov ? c.omb * (c.grad_scale * p.m.grad[i]) + c.beta * v : v;
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

// The momentum's update, and the sum of squares of 16,384 elements.
__global__ void __launch_bounds__(256) muon_norm_kernel(Group g) {
  __shared__ double sh[4];
  const int at = find_prob(g, blockIdx.x), block = (int)(blockIdx.x - g.first[at]);
  const Prob& p = g.p[at];
  const size_t n = (size_t)p.m.rows * p.m.cols, i0 = (size_t)block * kNormElems, i1 = min(n, i0 + kNormElems);
  double sum = 0.0;
  for (size_t i = i0 + threadIdx.x; i < i1; i += 256) {
    if (!p.m.src) p.m.moment[i] = g.c.beta * p.m.moment[i] + g.c.omb * (g.c.grad_scale * p.m.grad[i]);
    const double v = source_at(p, g.c, i);
    sum += v * v;
  }
  sum = wave_sum_f64(sum);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.part[block] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__global__ void __launch_bounds__(256) muon_scale_kernel(Group g) {
  __shared__ double sh[256];
  const Prob& p = g.p[blockIdx.x];
  const int blocks = (int)(((size_t)p.m.rows * p.m.cols + kNormElems - 1) / kNormElems);
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) sum += p.part[i];
  sh[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 128; o; o /= 2) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *p.scale = (float)((double)kXScale / (sqrt(sh[0]) + (double)g.c.eps));
}

// X = scale * source as two halves, zero in the padding.  A block takes a row's 2048 columns.
__global__ void __launch_bounds__(256) muon_split_kernel(Group g) {
  const int at = find_prob(g, blockIdx.x), block = (int)(blockIdx.x - g.first[at]);
  const Prob& p = g.p[at];
  const int per_row = (p.ld + 2047) / 2048, row = block / per_row, col = (block % per_row) * 2048 + threadIdx.x * 8;
  if (col >= p.ld) return;
  const float s = *p.scale;
  typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
  f16x8 h, l;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float v = row < p.m.rows && col + u < p.m.cols ? s * source_at(p, g.c, (size_t)row * p.m.cols + col + u) : 0.f;
    h[u] = (half_t)v;
    l[u] = (half_t)(v - (float)h[u]);
  }
  *(f16x8*)(p.xh[0] + (size_t)row * p.ld + col) = h;
  *(f16x8*)(p.xl[0] + (size_t)row * p.ld + col) = l;
}

#define MUON_SHARED(S)                                                \
  __shared__ __attribute__((aligned(16))) char la0[S::rows * 128];    \
  __shared__ __attribute__((aligned(16))) char lw0[S::cols * 128];    \
  __shared__ __attribute__((aligned(16))) char la1[S::rows * 128];    \
  __shared__ __attribute__((aligned(16))) char lw1[S::cols * 128];    \
  __shared__ __attribute__((aligned(16))) char lep[S::waves * 4096];

__device__ __forceinline__ uint16_t f16_bits(float v) { return __builtin_bit_cast(uint16_t, (half_t)v); }

// A symmetric tile: alpha * acc + beta * in (null: 0), stored at its place and, off the diagonal, mirrored.
template <typename S>
__device__ __forceinline__ void store_symmetric(pt_f32x16 (&acc)[S::NT][S::MT], const half_t* in, half_t* out, int ld, int tm, int tn,
                                                float alpha, float beta, char* lep) {
  constexpr int MT = S::MT;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hf = lane >> 5;
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = row0 + 32 * i + l32;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int col = col0 + pt_col(j, e, hf);
        float v = alpha * acc[j][i][e];
        // (the input is symmetric too: read across, where neighbouring lanes' values are neighbours)
        if (in && row < ld && col < ld) v += beta * (float)in[(size_t)col * ld + row];
        acc[j][i][e] = v;
        if (tm != tn && row < ld && col < ld) out[(size_t)col * ld + row] = (half_t)v;
      }
  }
  pt_hand_out_16<MT>(
      lep + wave * 4096, lane, [&](int j, int i, int e) { return f16_bits(acc[j][i][e]); },
      [&](int r, int c, pt_u32x4 v) {
        if (row0 + r < ld && col0 + c < ld) *(pt_u32x4*)(out + (size_t)(row0 + r) * ld + col0 + c) = v;
      });
}

// A = X X^T (the shorter side's), scaled
template <typename S>
__global__ void __launch_bounds__(64 * S::waves, 2) muon_gram_kernel(Group g, int cur) {
  MUON_SHARED(S)
  const int item = pt_item(g.items);
  if (item < 0) return;
  const int at = find_prob(g, item);
  const Prob& p = g.p[at];
  int tm, tn;
  pt_tile_triangle(item - (int)g.first[at], tm, tn);
  pt_f32x16 acc[S::NT][S::MT];
  const half_t* const x = p.xh[cur];
  if (p.m.rows > p.m.cols)
    pt_product<half_t, true, true, S>(x, p.ld, tm * S::rows, p.sp, x, p.ld, tn * S::cols, p.sp, 0, p.rp, la0, lw0, la1, lw1, acc);
  else
    pt_product<half_t, false, false, S>(x, p.ld, tm * S::rows, p.sp, x, p.ld, tn * S::cols, p.sp, 0, p.ld, la0, lw0, la1, lw1, acc);
  store_symmetric<S>(acc, nullptr, p.a, p.sp, tm, tn, kAScale / (kXScale * kXScale), 0.f, lep);
}

// B = b A + c A^2
template <typename S>
__global__ void __launch_bounds__(64 * S::waves, 2) muon_poly_kernel(Group g) {
  MUON_SHARED(S)
  const int item = pt_item(g.items);
  if (item < 0) return;
  const int at = find_prob(g, item);
  const Prob& p = g.p[at];
  int tm, tn;
  pt_tile_triangle(item - (int)g.first[at], tm, tn);
  pt_f32x16 acc[S::NT][S::MT];
  pt_product<half_t, false, false, S>(p.a, p.sp, tm * S::rows, p.sp, p.a, p.sp, tn * S::cols, p.sp, 0, p.sp, la0, lw0, la1, lw1, acc);
  store_symmetric<S>(acc, p.a, p.b, p.sp, tm, tn, kC / kAScale, kB, lep);
}

// X <- a X + B X, or after the last step what becomes of it
template <typename S>
__global__ void __launch_bounds__(64 * S::waves, 2) muon_update_kernel(Group g, int cur, int last) {
  MUON_SHARED(S)
  constexpr int MT = S::MT;
  const int item = pt_item(g.items);
  if (item < 0) return;
  const int at = find_prob(g, item);
  const Prob& p = g.p[at];
  int tm, tn;
  pt_tile_pos(item - (int)g.first[at], (p.rp + S::rows - 1) / S::rows, (p.ld + S::cols - 1) / S::cols, tm, tn);
  pt_f32x16 acc[2][MT];
  if (p.m.rows > p.m.cols)
    pt_product<half_t, false, false, S>(p.xh[cur], p.ld, tm * S::rows, p.rp, p.b, p.sp, tn * S::cols, p.sp, 0, p.sp, la0, lw0, la1,
                                        lw1, acc);
  else
    pt_product<half_t, false, true, S>(p.b, p.sp, tm * S::rows, p.sp, p.xh[cur], p.ld, tn * S::cols, p.ld, 0, p.sp, la0, lw0, la1,
                                       lw1, acc);
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = tm * S::rows + wave / S::WN * 32 * MT, col0 = tn * S::cols + wave % S::WN * 64;
  typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
  const int rows = p.m.rows, cols = p.m.cols;
  pt_hand_out_32<MT, 2>(
      lep + wave * 4096, lane, [&](int j, int i, int e) { return acc[j][i][e]; },
      [&](int r, int c, pt_f32x4 v) {
        const int row = row0 + r, col = col0 + c;
        if (row >= p.rp || col >= p.ld) return;
        const size_t i = (size_t)row * p.ld + col;
        const f16x4 h = *(const f16x4*)(p.xh[cur] + i), l = *(const f16x4*)(p.xl[cur] + i);
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = fmaf(v[u], 1.f / kAScale, kA * ((float)h[u] + (float)l[u]));
        if (!last) {
          f16x4 nh, nl;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            nh[u] = (half_t)v[u];
            nl[u] = (half_t)(v[u] - (float)nh[u]);
          }
          *(f16x4*)(p.xh[cur ^ 1] + i) = nh;
          *(f16x4*)(p.xl[cur ^ 1] + i) = nl;
          return;
        }
        if (row >= rows) return;
        const size_t o = (size_t)row * cols + col;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (col + u >= cols) break;
          const float x = v[u] * (1.f / kXScale);
          if (p.m.src) {
            p.m.out[o + u] = __builtin_bit_cast(uint16_t, (bfloat)x);
          } else {
            const float w = g.c.decay * p.m.param[o + u] - p.step * x;
            p.m.param[o + u] = w;
            if (p.m.param_bf16) p.m.param_bf16[o + u] = __builtin_bit_cast(uint16_t, (bfloat)w);
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
  size_t off = 0;
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
void number(Group& g, F items) {
  g.items = 0;
  for (int i = 0; i < g.count; ++i) {
    g.first[i] = g.items;
    g.items += (uint32_t)items(g.p[i]);
  }
}
int up(int n, int t) { return (n + t - 1) / t; }
int triangle(int n) { return n * (n + 1) / 2; }

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
    }
    number(g, [](const Prob& p) { return norm_blocks(p.m.rows, p.m.cols); });
    hipLaunchKernelGGL(muon_norm_kernel, dim3(g.items), dim3(256), 0, s, g);
    hipLaunchKernelGGL(muon_scale_kernel, dim3(g.count), dim3(256), 0, s, g);
    number(g, [](const Prob& p) { return p.rp * up(p.ld, 2048); });
    hipLaunchKernelGGL(muon_split_kernel, dim3(g.items), dim3(256), 0, s, g);
    for (int k = 0; k < c.steps; ++k) {
      const int cur = k & 1;
      number(g, [](const Prob& p) { return triangle(up(p.sp, PtMid::rows)); });
      hipLaunchKernelGGL(muon_gram_kernel<PtMid>, dim3(pt_grid(g.items)), dim3(64 * PtMid::waves), 0, s, g, cur);
      hipLaunchKernelGGL(muon_poly_kernel<PtMid>, dim3(pt_grid(g.items)), dim3(64 * PtMid::waves), 0, s, g);
      number(g, [](const Prob& p) { return up(p.rp, PtMid::rows) * up(p.ld, PtMid::cols); });
      hipLaunchKernelGGL(muon_update_kernel<PtMid>, dim3(pt_grid(g.items)), dim3(64 * PtMid::waves), 0, s, g, cur, k + 1 == c.steps);
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    from = to;
  }
  return hipSuccess;
}

}  // namespace rlhf
