// What lies between the projections and the attention calls on gfx950: RMS
// norm of each head and the rotation by its row's position (queries, keys,
// index queries and keys), the same on the way into the (paged) cache, and the
// backward of both.
//
// A head of D = 64 or 128 elements is one group of D / 8 lanes with 8 elements
// each.  A lane holds whole pairs of the rotation: in the half layout elements
// 4c .. 4c+3 and their partners R/2 further on, in pairs elements 8c .. 8c+7;
// so the rotation moves nothing between lanes, and the norm's sum of squares is
// the only exchange (3 or 4 DPP steps).  Angles: one CTA takes a tile of rows
// and forms the cosine and sine of every (row, pair) once, in LDS, for all
// heads and both tensors of the call; position times frequency and its
// reduction to a turn are in 64 bits (a position of 10^6 has fewer than 5 bits
// after the point left in 32), the cosine and sine of the reduced turn in 32.
// Everything between the bf16 input and the one rounding of the output is fp32.
//
// Large calls are bound by HBM: 39426 rows of 64 + 4 heads of 128 256 us,
// 5.3 TB/s, the backward of 32768 rows of 64 + 8 heads 346 us, 5.2 TB/s, every byte
// once.
// Small ones by a chain of latencies (launch, rows, angles, elements): 64 rows
// 4.3 us.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "msa_common.h"
#include "msa_profile.h"

namespace {

using namespace msa;

constexpr int kThreads = 256;
constexpr int kMaxRows = 32;             // rows per CTA at most
constexpr int kPer = 8;                  // elements per lane and head

// The rotation of one or several tensors, as the kernels take it.
struct Spec {
  const double* freq;                    // [pairs] radians per position
  int pairs;                             // rot_dim / 2; 0: no rotation
  int inter;                             // pairs (2i, 2i + 1) instead of (i, i + pairs)
  float scale;                           // on cosine and sine
  float sign;                            // -1: the transposed rotation (backward)
};

// E4M3 codes of y / scale: the scale as m / down, down a power of two and m from 1
// up to 2.
struct Code {
  int on;                                // 0: the output is bf16
  float down, m, inv_m;
};

// One tensor of a call: `heads` heads per row.
struct Part {
  const uint16_t* x;                     // bf16 rows, `stride` elements apart
  const uint16_t* g;                     // backward: gradient rows of the outputs, contiguous
  void* y;                               // output rows, `y_stride` elements apart
  const float* w;                        // norm weight, or null: no norm
  int64_t stride, y_stride;
  int heads;
  uint32_t magic;                        // ceil(2^32 / heads)
  int lg_lanes;                          // log2 of the lanes per head
  int spec;                              // which rotation, or -1
  Code code;
};

constexpr int kMaxParts = 3;
struct Parts {
  Part part[kMaxParts];
  Spec spec[2];
  int rows;                              // rows per CTA
  float eps;
};

__device__ __forceinline__ void unpack4(uint2 r, float (&f)[4]) {
  f[0] = __uint_as_float(r.x << 16);
  f[1] = __uint_as_float(r.x & 0xFFFF0000u);
  f[2] = __uint_as_float(r.y << 16);
  f[3] = __uint_as_float(r.y & 0xFFFF0000u);
}
__device__ __forceinline__ uint2 pack4(const float (&f)[4]) {
  return make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
}
// E4M3 codes of f / scale, to nearest even; beyond the format's range its largest
// value (the conversion alone would give NaN), NaN stays.  f * down is exact
// (unless its code is zero or the largest), and the quotient itself where the scale
// is a power of two.  Else f * down * inv_m alone is off by up to 1.5 steps of fp32,
// which takes 60 of the 65536 bf16 values across the middle between two codes at
// a scale of 0.4375; one step with the product's remainder, which fp32 holds, gives
// the rounded quotient (compared with the division for every bf16 mantissa and
// every m); it takes 30000 rows of 64 + 8 heads 190 us instead of 176.  q is bounded
// so that infinities leave no NaN.
__device__ __forceinline__ float to_range(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }
__device__ __forceinline__ uint32_t code4(const float (&f)[4], const Code& c) {
  float z[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) z[e] = f[e] * c.down;
  if (c.m != 1.f) {                      // the same for every lane
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float q = __builtin_amdgcn_fmed3f(z[e] * c.inv_m, -512.f, 512.f);
      z[e] = fmaf(-fmaf(q, c.m, -z[e]), c.inv_m, q);    // in this order -0 stays
    }
  }
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(to_range(z[0]), to_range(z[1]), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(to_range(z[2]), to_range(z[3]), r, true);
  return static_cast<uint32_t>(r);
}

// Sum over the lanes of a head (the same bits in each of them).
__device__ __forceinline__ float head_sum(float x, int lg_lanes) {
  auto add = [](float v, uint32_t o) { return v + __uint_as_float(o); };
  x = add(x, xor_lane_u32<1>(__float_as_uint(x)));
  x = add(x, xor_lane_u32<2>(__float_as_uint(x)));
  x = add(x, xor_lane_u32<4>(__float_as_uint(x)));
  if (lg_lanes == 4) x = add(x, xor_lane_u32<8>(__float_as_uint(x)));
  return x;
}

// A lane's elements of a head: a .. a+3 and b .. b+3, rotated by angles
// ang .. ang+3 (ang < 0: not rotated).
struct LaneDims {
  int a, b, ang;
};
__device__ __forceinline__ LaneDims lane_dims(const Part& pt, const Spec& sp) {
  const int c = threadIdx.x & ((1 << pt.lg_lanes) - 1);
  LaneDims d{kPer * c, kPer * c + 4, -1};
  if (pt.spec >= 0 && 4 * c < sp.pairs) {
    d.ang = 4 * c;
    if (!sp.inter) {
      d.a = 4 * c;
      d.b = sp.pairs + 4 * c;
    }
  }
  return d;
}

// (u, v) turned by the lane's four angles.
__device__ __forceinline__ void rotate(float (&u)[4], float (&v)[4], const float4& c, const float4& s, int inter) {
  auto turn = [](float& x, float& y, float cc, float ss) {
    const float a = fmaf(x, cc, -(y * ss)), b = fmaf(y, cc, x * ss);
    x = a;
    y = b;
  };
  if (inter) {
    turn(u[0], u[1], c.x, s.x);
    turn(u[2], u[3], c.y, s.y);
    turn(v[0], v[1], c.z, s.z);
    turn(v[2], v[3], c.w, s.w);
  } else {
    turn(u[0], v[0], c.x, s.x);
    turn(u[1], v[1], c.y, s.y);
    turn(u[2], v[2], c.z, s.z);
    turn(u[3], v[3], c.w, s.w);
  }
}

// Rows row0 .. row0 + n - 1 (n <= 64): position of each, or INT32_MIN for a
// row behind the last sequence; with `dst`, the cache row it goes to, or -1.
// One wave, one row per lane.
__device__ __forceinline__ void locate_rows(const msa_seqs& sq, int64_t row0, int n, int32_t* pos, int64_t* dst) {
  const int lane = lane_id();
  int lo = find_seq_wave(sq.q_offsets, sq.num_seqs, row0);
  int hi = n > 1 ? find_seq_wave(sq.q_offsets, sq.num_seqs, row0 + n - 1) : lo;
  const int64_t row = row0 + min(lane, n - 1);
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (static_cast<int64_t>(sq.q_offsets[mid]) <= row) lo = mid; else hi = mid - 1;
  }
  const int begin = sq.q_offsets[lo], rows = sq.q_offsets[lo + 1] - begin;
  const int t = static_cast<int>(row - begin);
  const int64_t p = static_cast<int64_t>(sq.kv_lens[lo]) - rows + t;
  const bool ours = t < rows;
  if (lane < n) pos[lane] = ours ? static_cast<int32_t>(p) : INT32_MIN;
  if (dst) {
    int64_t to = -1;
    if (ours && p >= 0) {
      if (sq.block_table) {
        const int shift = 31 - __clz(sq.page_size);
        if ((p >> shift) < sq.block_table_stride) {
          const int64_t page = sq.block_table[static_cast<int64_t>(lo) * sq.block_table_stride + (p >> shift)];
          if (page >= 0 && page < (sq.total_kv_rows >> shift)) to = (page << shift) + (p & (sq.page_size - 1));
        }
      } else {
        const int64_t at = sq.kv_starts[lo] + p;
        if (at >= 0 && at < sq.total_kv_rows) to = at;
      }
    }
    if (lane < n) dst[lane] = to;
  }
}

// Cosines and sines of n rows' angles: cs[row][2][pairs].
__device__ __forceinline__ void fill_angles(const Spec& sp, const int32_t* pos, int n, float* cs) {
  for (int i = threadIdx.x; i < n * sp.pairs; i += kThreads) {
    const int r = i / sp.pairs, j = i - r * sp.pairs;
    double turns = static_cast<double>(pos[r]) * sp.freq[j] * 0.15915494309189533577;   // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * static_cast<float>(turns), &s, &c);
    cs[(2 * r) * sp.pairs + j] = c * sp.scale;
    cs[(2 * r + 1) * sp.pairs + j] = s * (sp.scale * sp.sign);
  }
}

// The heads of one part in the CTA's rows: iteration `it` of the part takes
// heads (row, head) it * groups .. + groups - 1 of the flattened list, one per
// lane group; the CTA takes every `step`-th iteration from `it0` on.
template <bool CACHE>
__device__ __forceinline__ int run_part(const Part& pt, const Spec& sp, int64_t row0, int n, float eps, const int32_t* pos,
                                        const int64_t* dst, const float* cs, int it, int step) {
  const int group = threadIdx.x >> pt.lg_lanes, groups = kThreads >> pt.lg_lanes;
  const int total = n * pt.heads;
  const int iters = (total + groups - 1) / groups;
  const int D = kPer << pt.lg_lanes;
  const LaneDims d = lane_dims(pt, sp);
  float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
  if (pt.w) {
    const float* w = pt.w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      wa[e] = w[d.a + e];
      wb[e] = w[d.b + e];
    }
  }
  auto at = [&](int i, int* r, int* h) {
    const int idx = min(i * groups + group, total - 1);
    *r = static_cast<int>(__umulhi(static_cast<uint32_t>(idx), pt.magic));
    if (pt.heads == 1) *r = idx;
    *h = idx - *r * pt.heads;
  };
  auto load = [&](int i, uint2& xa, uint2& xb) {
    int r, h;
    at(i, &r, &h);
    const uint16_t* x = pt.x + (row0 + r) * pt.stride + h * D;
    xa = *reinterpret_cast<const uint2*>(x + d.a);
    xb = *reinterpret_cast<const uint2*>(x + d.b);
  };
  uint2 na{}, nb{};
  if (it < iters) load(it, na, nb);
  for (; it < iters; it += step) {
    const uint2 xa = na, xb = nb;
    if (it + step < iters) load(it + step, na, nb);
    int r, h;
    at(it, &r, &h);
    float u[4], v[4];
    unpack4(xa, u);
    unpack4(xb, v);
    if (pt.w) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) ss = fmaf(u[e], u[e], fmaf(v[e], v[e], ss));
      const float rstd = rsqrtf(head_sum(ss, pt.lg_lanes) * (pt.lg_lanes == 4 ? 1.f / 128 : 1.f / 64) + eps);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u[e] = u[e] * rstd * wa[e];
        v[e] = v[e] * rstd * wb[e];
      }
    }
    if (d.ang >= 0) {
      const float* c = cs + 2 * r * sp.pairs + d.ang;
      rotate(u, v, *reinterpret_cast<const float4*>(c), *reinterpret_cast<const float4*>(c + sp.pairs), sp.inter);
    }
    const bool keep = it * groups + group < total && (CACHE ? dst[r] >= 0 : pos[r] != INT32_MIN);
    if (keep) {
      const int64_t to = (CACHE ? dst[r] : row0 + r) * pt.y_stride + h * D;
      if (pt.code.on) {
        uint8_t* y = static_cast<uint8_t*>(pt.y) + to;
        *reinterpret_cast<uint32_t*>(y + d.a) = code4(u, pt.code);
        *reinterpret_cast<uint32_t*>(y + d.b) = code4(v, pt.code);
      } else {
        // elements that nothing is applied to keep their bits (NaN payloads too)
        const bool same = !pt.w && d.ang < 0;
        uint16_t* y = static_cast<uint16_t*>(pt.y) + to;
        *reinterpret_cast<uint2*>(y + d.a) = same ? xa : pack4(u);
        *reinterpret_cast<uint2*>(y + d.b) = same ? xb : pack4(v);
      }
    }
  }
  return it - iters;                     // the CTA's first iteration of the next part
}

// LDS: angles of each rotation, [rows][2][pairs].
template <int NPARTS, bool CACHE>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(Parts a, msa_seqs sq) {
  extern __shared__ __align__(16) float cs[];
  __shared__ int32_t pos[kMaxRows];
  __shared__ int64_t dst[kMaxRows];
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows;
  const int n = static_cast<int>(min(static_cast<int64_t>(a.rows), sq.total_q_rows - row0));
  if (threadIdx.x < kWave) locate_rows(sq, row0, n, pos, CACHE ? dst : nullptr);
  __syncthreads();
  float* cs1 = cs + a.rows * 2 * a.spec[0].pairs;
  fill_angles(a.spec[0], pos, n, cs);
  if (CACHE) fill_angles(a.spec[1], pos, n, cs1);
  __syncthreads();
  int it = blockIdx.y;
#pragma unroll
  for (int i = 0; i < NPARTS; ++i) {
    const bool second = CACHE && a.part[i].spec == 1;
    it = run_part<CACHE>(a.part[i], second ? a.spec[1] : a.spec[0], row0, n, a.eps, pos, dst, second ? cs1 : cs, it,
                         gridDim.y);
  }
}

// ---------------------------------------------------------------- backward
constexpr int kGradCtas = 1024;          // CTAs at most: partial weight gradients of each

// h = R^T g; with the norm, xh = x rstd, m = mean(h w xh):
//   d x = rstd (h w - xh m),  d w = sum over rows and heads of h xh.
// Each lane sums its 8 elements' d w over the heads it takes; the CTA's lane
// groups are added in LDS in their order, and the CTAs by norm_grad_kernel.
__device__ __forceinline__ void run_part_back(const Part& pt, const Spec& sp, int64_t row0, int n, float eps, const int32_t* pos,
                                              const float* cs, float (&dwa)[4], float (&dwb)[4]) {
  const int group = threadIdx.x >> pt.lg_lanes, groups = kThreads >> pt.lg_lanes;
  const int total = n * pt.heads;
  const int iters = (total + groups - 1) / groups;
  const int D = kPer << pt.lg_lanes;
  const LaneDims d = lane_dims(pt, sp);
  float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
  if (pt.w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      wa[e] = pt.w[d.a + e];
      wb[e] = pt.w[d.b + e];
    }
  }
  auto at = [&](int i, int* r, int* h) {
    const int idx = min(i * groups + group, total - 1);
    *r = static_cast<int>(__umulhi(static_cast<uint32_t>(idx), pt.magic));
    if (pt.heads == 1) *r = idx;
    *h = idx - *r * pt.heads;
  };
  struct Raw4 {
    uint2 xa, xb, ga, gb;
  };
  auto load = [&](int i, Raw4& o) {
    int r, h;
    at(i, &r, &h);
    const uint16_t* g = pt.g + ((row0 + r) * pt.heads + h) * D;
    o.ga = *reinterpret_cast<const uint2*>(g + d.a);
    o.gb = *reinterpret_cast<const uint2*>(g + d.b);
    if (pt.w) {
      const uint16_t* x = pt.x + (row0 + r) * pt.stride + h * D;
      o.xa = *reinterpret_cast<const uint2*>(x + d.a);
      o.xb = *reinterpret_cast<const uint2*>(x + d.b);
    }
  };
  Raw4 next{};
  if (iters > 0) load(0, next);
  for (int it = 0; it < iters; ++it) {
    const Raw4 cur = next;
    if (it + 1 < iters) load(it + 1, next);
    int r, h;
    at(it, &r, &h);
    const bool keep = it * groups + group < total && pos[r] != INT32_MIN;
    float u[4], v[4];
    unpack4(cur.ga, u);
    unpack4(cur.gb, v);
    if (d.ang >= 0) {
      const float* c = cs + 2 * r * sp.pairs + d.ang;
      rotate(u, v, *reinterpret_cast<const float4*>(c), *reinterpret_cast<const float4*>(c + sp.pairs), sp.inter);
    }
    if (pt.w) {
      float xu[4], xv[4];
      unpack4(cur.xa, xu);
      unpack4(cur.xb, xv);
      const float inv_d = pt.lg_lanes == 4 ? 1.f / 128 : 1.f / 64;
      float ss = 0.f, dot = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ss = fmaf(xu[e], xu[e], fmaf(xv[e], xv[e], ss));
        dot = fmaf(u[e] * wa[e], xu[e], fmaf(v[e] * wb[e], xv[e], dot));
      }
      const float rstd = rsqrtf(head_sum(ss, pt.lg_lanes) * inv_d + eps);
      const float m = head_sum(dot, pt.lg_lanes) * rstd * inv_d;     // mean(h w xh)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float hu = xu[e] * rstd, hv = xv[e] * rstd;
        if (keep) {
          dwa[e] = fmaf(u[e], hu, dwa[e]);
          dwb[e] = fmaf(v[e], hv, dwb[e]);
        }
        u[e] = rstd * fmaf(u[e], wa[e], -(hu * m));
        v[e] = rstd * fmaf(v[e], wb[e], -(hv * m));
      }
    }
    if (keep) {
      uint16_t* y = static_cast<uint16_t*>(pt.y) + (row0 + r) * pt.y_stride + h * D;
      *reinterpret_cast<uint2*>(y + d.a) = pack4(u);
      *reinterpret_cast<uint2*>(y + d.b) = pack4(v);
    }
  }
}

__global__ __launch_bounds__(kThreads) void norm_rope_backward_kernel(Parts a, msa_seqs sq, float* dw_part) {
  extern __shared__ __align__(16) float cs[];
  __shared__ int32_t pos[kMaxRows];
  __shared__ __align__(16) float red[kThreads * kPer];
  float dw[2][2][4] = {};
  const int64_t tiles = (sq.total_q_rows + a.rows - 1) / a.rows;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row0 = tile * a.rows;
    const int n = static_cast<int>(min(static_cast<int64_t>(a.rows), sq.total_q_rows - row0));
    __syncthreads();                     // the last tile's angles are read
    if (threadIdx.x < kWave) locate_rows(sq, row0, n, pos, nullptr);
    __syncthreads();
    fill_angles(a.spec[0], pos, n, cs);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (a.part[i].heads > 0) run_part_back(a.part[i], a.spec[0], row0, n, a.eps, pos, cs, dw[i][0], dw[i][1]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (a.part[i].heads == 0 || !a.part[i].w) continue;
    const Part& pt = a.part[i];
    const LaneDims d = lane_dims(pt, a.spec[0]);
    const int D = kPer << pt.lg_lanes, groups = kThreads >> pt.lg_lanes;
    __syncthreads();
    float* mine = red + (threadIdx.x >> pt.lg_lanes) * D;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mine[d.a + e] = dw[i][0][e];
      mine[d.b + e] = dw[i][1][e];
    }
    __syncthreads();
    if (threadIdx.x < D) {
      float sum = 0.f;
      for (int gidx = 0; gidx < groups; ++gidx) sum += red[gidx * D + threadIdx.x];
      dw_part[(static_cast<int64_t>(blockIdx.x) * 2 + i) * D + threadIdx.x] = sum;
    }
  }
}

// d w = sum of the CTAs' partials (a tensor without heads has none): a CTA takes
// 16 elements, 64 threads each, which are added in a fixed order.  (16 threads per
// element, whose 64 reads waited for one another, took 20 us.)
constexpr int kGradThreads = 1024;
__global__ __launch_bounds__(kGradThreads) void norm_grad_kernel(const float* __restrict__ dw_part, int q_ctas,
                                                                 int k_ctas, int D, float* dq_w, float* dk_w) {
  constexpr int kRows = kGradThreads / 16, kBatch = 4;
  __shared__ float red[kRows][17];
  const int i = blockIdx.y;
  float* out = i ? dk_w : dq_w;
  const int ctas = i ? k_ctas : q_ctas;
  if (!out) return;                      // uniform over the CTA
  const int e = threadIdx.x & 15, j = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + e;
  float sum = 0.f;
  for (int c0 = j; c0 < ctas; c0 += kRows * kBatch) {
    float x[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int c = c0 + u * kRows;
      x[u] = dw_part[(static_cast<int64_t>(min(c, ctas - 1)) * 2 + i) * D + col];
      x[u] = c < ctas ? x[u] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) sum += x[u];
  }
  red[j][e] = sum;
  __syncthreads();
#pragma unroll
  for (int d = kRows / 2; d > 0; d /= 2) {
    if (j < d) red[j][e] += red[j + d][e];
    __syncthreads();
  }
  if (j == 0) out[col] = red[0][e];
}

// ---------------------------------------------------------------- latent cache rows
// A row of the latent cache: the norm of the token's latent (R elements, a wave
// with R / 64 each) and its shared key part, rotated (64 elements, one pair for
// each of 32 lanes).  A wave takes two rows at a time, since one row's pairs would
// leave half of its lanes idle through the angles' sines, the longest part of the
// arithmetic; their elements are requested before the rows are located.
template <int R>
__global__ __launch_bounds__(kThreads) void latent_append_kernel(const uint16_t* __restrict__ latent, int64_t latent_stride,
                                                                 const uint16_t* __restrict__ k_rope, int64_t k_rope_stride,
                                                                 const float* __restrict__ weight, float eps, Spec sp, Code code,
                                                                 msa_seqs sq, int rows, void* __restrict__ cache) {
  constexpr int kRot = 64, N = R / kWave;
  __shared__ int32_t pos[kMaxRows];
  __shared__ int64_t dst[kMaxRows];
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows;
  const int n = static_cast<int>(min(static_cast<int64_t>(rows), sq.total_q_rows - row0));
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  // the lane's pair of row r + lane / 32: rotated ones first, then the rest of the part
  const int i = lane & 31, mine = lane >> 5;
  const bool turned = i < sp.pairs;
  const int a = !turned ? 2 * i : sp.inter ? 2 * i : i;
  const int b = !turned || sp.inter ? a + 1 : sp.pairs + i;
  constexpr int kStep = 2 * kThreads / kWave;
  uint2 x[2][2];                         // 8 or 4 elements of each row
  uint32_t ka = 0, kb = 0;
  auto load = [&](int r) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {        // a row past the CTA's last is its last again
      const uint16_t* src = latent + (row0 + min(r + j, n - 1)) * latent_stride + N * lane;
      x[j][0] = *reinterpret_cast<const uint2*>(src);
      if constexpr (N == 8) x[j][1] = *reinterpret_cast<const uint2*>(src + 4);
    }
    const uint16_t* kr = k_rope + (row0 + min(r + mine, n - 1)) * k_rope_stride;
    ka = kr[a];
    kb = kr[b];
  };
  int r = 2 * wave;
  if (r < n) load(r);
  if (threadIdx.x < kWave) locate_rows(sq, row0, n, pos, dst);
  float w[N];
#pragma unroll
  for (int c = 0; c < N; ++c) w[c] = weight ? weight[N * lane + c] : 1.f;
  const double freq = turned ? sp.freq[i] : 0.0;
  __syncthreads();
  for (; r < n; r += kStep) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t to = r + j < n ? dst[r + j] : -1;
      if (to < 0) continue;              // the same in every lane
      float u[4], v[4] = {};
      unpack4(x[j][0], u);
      if constexpr (N == 8) unpack4(x[j][1], v);
      if (weight) {
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) ss = fmaf(u[c], u[c], fmaf(v[c], v[c], ss));
        ss = head_sum(ss, 4);
        ss += __uint_as_float(xor_lane_u32<16>(__float_as_uint(ss)));
        ss += __uint_as_float(xor_lane_u32<32>(__float_as_uint(ss)));
        const float rstd = rsqrtf(ss * (1.f / R) + eps);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u[c] = u[c] * rstd * w[c];
          if constexpr (N == 8) v[c] = v[c] * rstd * w[4 + c];
        }
      }
      const int64_t at = to * (R + kRot) + N * lane;
      if (code.on) {
        uint8_t* y = static_cast<uint8_t*>(cache) + at;
        *reinterpret_cast<uint32_t*>(y) = code4(u, code);
        if constexpr (N == 8) *reinterpret_cast<uint32_t*>(y + 4) = code4(v, code);
      } else {
        // elements that nothing is applied to keep their bits (NaN payloads too)
        uint16_t* y = static_cast<uint16_t*>(cache) + at;
        *reinterpret_cast<uint2*>(y) = weight ? pack4(u) : x[j][0];
        if constexpr (N == 8) *reinterpret_cast<uint2*>(y + 4) = weight ? pack4(v) : x[j][1];
      }
    }
    const int rr = r + mine;
    const int64_t to = rr < n ? dst[rr] : -1;
    if (to >= 0) {
      float ra = __uint_as_float(ka << 16), rb = __uint_as_float(kb << 16);
      if (turned) {
        double turns = static_cast<double>(pos[rr]) * freq * 0.15915494309189533577;   // 1 / (2 pi)
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * static_cast<float>(turns), &s, &c);
        c *= sp.scale;
        s *= sp.scale;
        const float y = fmaf(ra, c, -(rb * s));
        rb = fmaf(rb, c, ra * s);
        ra = y;
      }
      const int64_t at = to * (R + kRot) + R;
      if (code.on) {
        const float pair[4] = {ra, rb, 0.f, 0.f};
        const uint32_t cd = code4(pair, code);
        uint8_t* y = static_cast<uint8_t*>(cache) + at;
        y[a] = static_cast<uint8_t>(cd);
        y[b] = static_cast<uint8_t>(cd >> 8);
      } else {
        const uint32_t pr = turned ? pack_bf16x2(ra, rb) : (ka | (kb << 16));
        uint16_t* y = static_cast<uint16_t*>(cache) + at;
        y[a] = static_cast<uint16_t>(pr);
        y[b] = static_cast<uint16_t>(pr >> 16);
      }
    }
    if (r + kStep < n) load(r + kStep);
  }
}

// ---------------------------------------------------------------- host side
int validate_rope(const msa_rope* r, int dim) {
  if (!r || r->rot_dim == 0) return MSA_OK;
  if (r->rot_dim < 0 || r->rot_dim > dim || !r->inv_freq) return MSA_ERR_INVALID;
  if (!(r->scale > -3.0e38f && r->scale < 3.0e38f)) return MSA_ERR_INVALID;
  if (r->rot_dim % 8 != 0) return MSA_ERR_UNSUPPORTED;
  return MSA_OK;
}
Spec spec_of(const msa_rope* r, bool inverse = false) {
  if (!r || r->rot_dim == 0) return Spec{nullptr, 0, 0, 1.f, 1.f};
  return Spec{r->inv_freq, r->rot_dim / 2, r->interleaved != 0, r->scale, inverse ? -1.f : 1.f};
}

bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }

// A tensor of rows of `heads` heads: null exactly if it has no heads; rows do
// not overlap, and pieces of 4 elements are aligned.
int check_rows(const void* x, int64_t stride, int heads, int dim) {
  if (heads == 0) return MSA_OK;
  if (!x || stride < static_cast<int64_t>(heads) * dim) return MSA_ERR_INVALID;
  if (!aligned8(x) || stride % 4 != 0) return MSA_ERR_UNSUPPORTED;
  return MSA_OK;
}

int lg_lanes(int dim) { return dim == 128 ? 4 : 3; }

Part part_of(const void* x, int64_t stride, int heads, int dim, const float* w, void* y, int64_t y_stride, int spec) {
  Part p{};
  p.x = static_cast<const uint16_t*>(x);
  p.y = y;
  p.w = w;
  p.stride = stride;
  p.y_stride = y_stride;
  p.heads = heads;
  p.magic = heads > 0 ? static_cast<uint32_t>(((uint64_t(1) << 32) + heads - 1) / heads) : 0;
  p.lg_lanes = lg_lanes(dim);
  p.spec = spec;
  return p;
}

// Iterations of a CTA over `rows` rows.
int64_t iterations(const Parts& a, int nparts, int64_t rows) {
  int64_t n = 0;
  for (int i = 0; i < nparts; ++i) {
    const int groups = kThreads >> a.part[i].lg_lanes;
    n += (rows * a.part[i].heads + groups - 1) / groups;
  }
  return n;
}

// Rows per CTA: enough for 8 iterations, which share the angles, the search for the
// rows' sequences and the weights, while there are more than `ctas` CTAs.  39426 rows
// of 64 + 4 heads take 256 us, and the backward of 32768 rows of 64 + 8 heads 346;
// with 4 iterations 277 and 378, with 16 263 and 351.  Forward: 2048 CTAs, eight per
// CU, which run at once (3929 rows of 64 + 4 heads into E4M3 24.7 us; with 1024 26.4,
// with 4096 26.0).
constexpr int kCtas = 2048;
int rows_per_cta(const Parts& a, int nparts, int64_t total, int ctas) {
  int rows = 1;
  while (rows < kMaxRows && iterations(a, nparts, rows) < 8 && (total + rows - 1) / rows > ctas) rows *= 2;
  return rows;
}

size_t angle_bytes(const Parts& a) { return sizeof(float) * 2 * a.rows * (a.spec[0].pairs + a.spec[1].pairs); }

template <int NPARTS, bool CACHE>
int launch_forward(const char* name, Parts a, const msa_seqs* seqs, hipStream_t stream) {
  a.rows = rows_per_cta(a, NPARTS, seqs->total_q_rows, kCtas);
  const int64_t tiles = (seqs->total_q_rows + a.rows - 1) / a.rows;
  if (tiles >= (int64_t(1) << 24)) return MSA_ERR_UNSUPPORTED;   // a grid's limit
  // few rows: a row's iterations go to several CTAs, up to 1024 in all
  int64_t split = std::min<int64_t>(iterations(a, NPARTS, a.rows), std::max<int64_t>(1, 1024 / tiles));
  msa_prof::launch(name, norm_rope_kernel<NPARTS, CACHE>, dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(split)),
                   dim3(kThreads), angle_bytes(a), stream, a, *seqs);
  return msa_host::launch_status();
}

// Positive, and its power of two has a normal reciprocal.
bool scale_ok(float x) { return x >= FLT_MIN && x <= 1.f / FLT_MIN; }
Code code_of(float scale) {
  int e;
  const float m = 2.f * std::frexp(scale, &e);           // scale = m 2^(e - 1)
  return Code{1, std::ldexp(1.f, 1 - e), m, 1.f / m};
}

int validate_heads(const msa_seqs* seqs, int H_q, int H_kv, int dim, float eps, const msa_rope* rope) {
  int st = msa_host::validate_seqs(seqs);
  if (st != MSA_OK) return st;
  if (H_q < 0 || H_kv < 0 || H_q + H_kv < 1 || dim < 1) return MSA_ERR_INVALID;
  if (!(eps >= 0.f && eps < 3.0e38f)) return MSA_ERR_INVALID;
  if (dim != 64 && dim != 128) return MSA_ERR_UNSUPPORTED;
  if (H_q > 1024 || H_kv > 1024) return MSA_ERR_UNSUPPORTED;
  return validate_rope(rope, dim);
}

int norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, bool fp8, float q_scale, float k_scale,
              const msa_seqs* seqs, int H_q, int H_kv, int dim, const float* q_weight, const float* k_weight, float eps,
              const msa_rope* rope, void* q_out, void* k_out, hipStream_t stream) {
  int st = validate_heads(seqs, H_q, H_kv, dim, eps, rope);
  if (st != MSA_OK) return st;
  if (fp8 && (!scale_ok(q_scale) || !scale_ok(k_scale))) return MSA_ERR_INVALID;
  if (seqs->total_q_rows == 0) return MSA_OK;
  if ((st = check_rows(q, q_stride, H_q, dim)) != MSA_OK) return st;
  if ((st = check_rows(k, k_stride, H_kv, dim)) != MSA_OK) return st;
  if ((H_q > 0 && !q_out) || (H_kv > 0 && !k_out)) return MSA_ERR_INVALID;
  if (!aligned8(q_out) || !aligned8(k_out)) return MSA_ERR_UNSUPPORTED;
  Parts a{};
  a.spec[0] = spec_of(rope);
  a.eps = eps;
  const int spec = a.spec[0].pairs > 0 ? 0 : -1;
  int n = 0;
  auto add = [&](const void* x, int64_t stride, int heads, const float* w, void* y, float scale) {
    if (heads == 0) return;
    a.part[n] = part_of(x, stride, heads, dim, w, y, static_cast<int64_t>(heads) * dim, spec);
    if (fp8) a.part[n].code = code_of(scale);
    ++n;
  };
  add(q, q_stride, H_q, q_weight, q_out, q_scale);
  add(k, k_stride, H_kv, k_weight, k_out, k_scale);
  return n == 2 ? launch_forward<2, false>("norm_rope_kernel", a, seqs, stream)
                : launch_forward<1, false>("norm_rope_kernel", a, seqs, stream);
}

int kv_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, bool fp8, float k_scale, float v_scale,
              const void* index_k, int64_t index_k_stride, const msa_seqs* seqs, int H_kv, int head_dim, int d_idx,
              const float* k_weight, const float* index_k_weight, float eps, const msa_rope* rope, const msa_rope* index_rope,
              void* k_cache, void* v_cache, void* index_k_cache, hipStream_t stream) {
  int st = validate_heads(seqs, H_kv, 0, head_dim, eps, rope);
  if (st != MSA_OK) return st;
  if (head_dim != 128 || H_kv > 64) return MSA_ERR_UNSUPPORTED;
  const bool with_index = index_k != nullptr || index_k_cache != nullptr;
  if (with_index) {
    if (!index_k || !index_k_cache) return MSA_ERR_INVALID;
    if (d_idx != 64 && d_idx != 128) return MSA_ERR_UNSUPPORTED;
    if ((st = validate_rope(index_rope, d_idx)) != MSA_OK) return st;
  }
  if (fp8 && (!scale_ok(k_scale) || !scale_ok(v_scale))) return MSA_ERR_INVALID;
  if (seqs->block_table && !(msa_host::is_pow2(seqs->page_size) && seqs->page_size >= 16 && seqs->page_size <= 8192))
    return MSA_ERR_INVALID;
  if (seqs->total_q_rows == 0) return MSA_OK;
  if ((st = check_rows(k, k_stride, H_kv, head_dim)) != MSA_OK) return st;
  if ((st = check_rows(v, v_stride, H_kv, head_dim)) != MSA_OK) return st;
  if (!k_cache || !v_cache) return MSA_ERR_INVALID;
  if (with_index && (st = check_rows(index_k, index_k_stride, 1, d_idx)) != MSA_OK) return st;
  if (!aligned8(k_cache) || !aligned8(v_cache) || !aligned8(index_k_cache)) return MSA_ERR_UNSUPPORTED;
  Parts a{};
  a.spec[0] = spec_of(rope);
  a.spec[1] = spec_of(with_index ? index_rope : nullptr);
  a.eps = eps;
  const int64_t row = static_cast<int64_t>(H_kv) * head_dim;
  a.part[0] = part_of(k, k_stride, H_kv, head_dim, k_weight, k_cache, row, a.spec[0].pairs > 0 ? 0 : -1);
  a.part[1] = part_of(v, v_stride, H_kv, head_dim, nullptr, v_cache, row, -1);
  if (fp8) {
    a.part[0].code = code_of(k_scale);
    a.part[1].code = code_of(v_scale);
  }
  if (!with_index) return launch_forward<2, true>("kv_append_kernel", a, seqs, stream);
  a.part[2] = part_of(index_k, index_k_stride, 1, d_idx, index_k_weight, index_k_cache, d_idx, a.spec[1].pairs > 0 ? 1 : -1);
  return launch_forward<3, true>("kv_append_kernel", a, seqs, stream);
}

// Rows per CTA: the smallest power of two, up to kMaxRows, that leaves at most 512 CTAs.
// Rows are located once per CTA, so few CTAs are best: 512 take 13.5 us for 18000 rows
// of 512 elements into E4M3 (launch and events included), 1024 14.2, 2048 16.4, 4096 24.
// As a call among others 11.4 us, into bf16 11.0 (5.3 and 7.1 at the rate of a large copy).
constexpr int64_t kLatentCtas = 512;
int latent_append(const void* latent, int64_t latent_stride, const void* k_rope, int64_t k_rope_stride, bool fp8, float scale,
                  const msa_seqs* seqs, int R, const float* weight, float eps, const msa_rope* rope, void* cache,
                  hipStream_t stream) {
  int st = msa_host::validate_seqs(seqs);
  if (st != MSA_OK) return st;
  if (R < 1 || !(eps >= 0.f && eps < 3.0e38f)) return MSA_ERR_INVALID;
  if (R != 256 && R != 512) return MSA_ERR_UNSUPPORTED;
  if ((st = validate_rope(rope, 64)) != MSA_OK) return st;
  if (fp8 && !scale_ok(scale)) return MSA_ERR_INVALID;
  if (seqs->block_table && !(msa_host::is_pow2(seqs->page_size) && seqs->page_size >= 16 && seqs->page_size <= 8192))
    return MSA_ERR_INVALID;
  if (seqs->total_q_rows == 0) return MSA_OK;
  if ((st = check_rows(latent, latent_stride, 1, R)) != MSA_OK) return st;
  if ((st = check_rows(k_rope, k_rope_stride, 1, 64)) != MSA_OK) return st;
  if (!cache) return MSA_ERR_INVALID;
  if (!aligned8(cache)) return MSA_ERR_UNSUPPORTED;
  const int64_t total = seqs->total_q_rows;
  int rows = 1;
  while (rows < kMaxRows && (total + rows - 1) / rows > kLatentCtas) rows *= 2;
  const int64_t ctas = (total + rows - 1) / rows;
  if (ctas >= (int64_t(1) << 24)) return MSA_ERR_UNSUPPORTED;          // a grid's limit
  const Code code = fp8 ? code_of(scale) : Code{};
  msa_prof::launch("latent_append_kernel", R == 512 ? latent_append_kernel<512> : latent_append_kernel<256>,
                   dim3(static_cast<unsigned>(ctas)), dim3(kThreads), 0, stream, static_cast<const uint16_t*>(latent),
                   latent_stride, static_cast<const uint16_t*>(k_rope), k_rope_stride, weight, eps, spec_of(rope), code, *seqs,
                   rows, cache);
  return msa_host::launch_status();
}

int64_t grad_ctas(const msa_seqs* seqs, const Parts& a) {
  return std::min<int64_t>(kGradCtas, (seqs->total_q_rows + a.rows - 1) / a.rows);
}

}  // namespace

extern "C" int msa_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const msa_seqs* seqs,
                                int num_q_heads, int num_kv_heads, int head_dim, const float* q_weight,
                                const float* k_weight, float eps, const msa_rope* rope, void* q_out, void* k_out,
                                hipStream_t stream) {
  return norm_rope(q, q_stride, k, k_stride, false, 1.f, 1.f, seqs, num_q_heads, num_kv_heads, head_dim, q_weight, k_weight,
                   eps, rope, q_out, k_out, stream);
}

extern "C" int msa_qk_norm_rope_fp8(const void* q, int64_t q_stride, const void* k, int64_t k_stride, float q_scale,
                                    float k_scale, const msa_seqs* seqs, int num_q_heads, int num_kv_heads, int head_dim,
                                    const float* q_weight, const float* k_weight, float eps, const msa_rope* rope,
                                    void* q_out, void* k_out, hipStream_t stream) {
  return norm_rope(q, q_stride, k, k_stride, true, q_scale, k_scale, seqs, num_q_heads, num_kv_heads, head_dim, q_weight,
                   k_weight, eps, rope, q_out, k_out, stream);
}

extern "C" size_t msa_qk_norm_rope_backward_workspace_size(const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                                                          int head_dim) {
  if (validate_heads(seqs, num_q_heads, num_kv_heads, head_dim, 0.f, nullptr) != MSA_OK) return 0;
  return sizeof(float) * 2 * head_dim * std::min<int64_t>(kGradCtas, std::max<int64_t>(1, seqs->total_q_rows));
}

extern "C" int msa_qk_norm_rope_backward(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                         const void* d_q_out, const void* d_k_out, const msa_seqs* seqs, int num_q_heads,
                                         int num_kv_heads, int head_dim, const float* q_weight, const float* k_weight,
                                         float eps, const msa_rope* rope, void* d_q, int64_t d_q_stride, void* d_k,
                                         int64_t d_k_stride, float* d_q_weight, float* d_k_weight, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream) {
  int st = validate_heads(seqs, num_q_heads, num_kv_heads, head_dim, eps, rope);
  if (st != MSA_OK) return st;
  if ((d_q_weight && !q_weight) || (d_k_weight && !k_weight)) return MSA_ERR_INVALID;
  const bool norms = (num_q_heads > 0 && q_weight) || (num_kv_heads > 0 && k_weight);
  Parts a{};
  a.spec[0] = spec_of(rope, true);
  a.eps = eps;
  const int spec = a.spec[0].pairs > 0 ? 0 : -1;
  struct In {
    const void* x;
    int64_t stride;
    const void* g;
    int heads;
    const float* w;
    void* d;
    int64_t d_stride;
  } in[2] = {{q, q_stride, d_q_out, num_q_heads, q_weight, d_q, d_q_stride},
             {k, k_stride, d_k_out, num_kv_heads, k_weight, d_k, d_k_stride}};
  if (seqs->total_q_rows > 0)
    for (const In& t : in) {
      if (t.heads == 0) continue;
      const int64_t packed = static_cast<int64_t>(t.heads) * head_dim;
      if (t.w && (st = check_rows(t.x, t.stride, t.heads, head_dim)) != MSA_OK) return st;
      if ((st = check_rows(t.g, packed, t.heads, head_dim)) != MSA_OK) return st;
      if ((st = check_rows(t.d, t.d_stride, t.heads, head_dim)) != MSA_OK) return st;
    }
  const size_t need = norms ? msa_qk_norm_rope_backward_workspace_size(seqs, num_q_heads, num_kv_heads, head_dim) : 0;
  if (norms && (!workspace || workspace_bytes < need)) return MSA_ERR_WORKSPACE;
  if (norms && !aligned8(workspace)) return MSA_ERR_UNSUPPORTED;
  int64_t ctas = 0;
  auto* part = static_cast<float*>(workspace);
  if (norms) {
    for (int i = 0; i < 2; ++i) {
      a.part[i] = part_of(in[i].x, in[i].stride, in[i].heads, head_dim, in[i].w, in[i].d, in[i].d_stride, spec);
      a.part[i].g = static_cast<const uint16_t*>(in[i].g);
    }
    a.rows = rows_per_cta(a, 2, seqs->total_q_rows, kGradCtas);
    ctas = grad_ctas(seqs, a);
    if (ctas > 0)
      msa_prof::launch("norm_rope_backward_kernel", norm_rope_backward_kernel, dim3(static_cast<unsigned>(ctas)),
                       dim3(kThreads), angle_bytes(a), stream, a, *seqs, part);
  } else if (seqs->total_q_rows > 0) {   // the transposed rotation alone
    int n = 0;
    for (const In& t : in)
      if (t.heads > 0)
        a.part[n++] = part_of(t.g, static_cast<int64_t>(t.heads) * head_dim, t.heads, head_dim, nullptr, t.d, t.d_stride, spec);
    st = n == 2 ? launch_forward<2, false>("norm_rope_kernel", a, seqs, stream)
                : launch_forward<1, false>("norm_rope_kernel", a, seqs, stream);
    if (st != MSA_OK) return st;
  }
  if (d_q_weight || d_k_weight)
    msa_prof::launch("norm_grad_kernel", norm_grad_kernel, dim3(head_dim / 16, 2), dim3(kGradThreads), 0, stream,
                     static_cast<const float*>(part), static_cast<int>(num_q_heads > 0 ? ctas : 0),
                     static_cast<int>(num_kv_heads > 0 ? ctas : 0), head_dim, d_q_weight, d_k_weight);
  return msa_host::launch_status();
}

extern "C" int msa_kv_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* index_k,
                             int64_t index_k_stride, const msa_seqs* seqs, int num_kv_heads, int head_dim, int d_idx,
                             const float* k_weight, const float* index_k_weight, float eps, const msa_rope* rope,
                             const msa_rope* index_rope, void* k_cache, void* v_cache, void* index_k_cache,
                             hipStream_t stream) {
  return kv_append(k, k_stride, v, v_stride, false, 1.f, 1.f, index_k, index_k_stride, seqs, num_kv_heads, head_dim, d_idx,
                   k_weight, index_k_weight, eps, rope, index_rope, k_cache, v_cache, index_k_cache, stream);
}

extern "C" int msa_kv_append_fp8(const void* k, int64_t k_stride, const void* v, int64_t v_stride, float k_scale,
                                 float v_scale, const void* index_k, int64_t index_k_stride, const msa_seqs* seqs,
                                 int num_kv_heads, int head_dim, int d_idx, const float* k_weight,
                                 const float* index_k_weight, float eps, const msa_rope* rope, const msa_rope* index_rope,
                                 void* k_cache, void* v_cache, void* index_k_cache, hipStream_t stream) {
  return kv_append(k, k_stride, v, v_stride, true, k_scale, v_scale, index_k, index_k_stride, seqs, num_kv_heads, head_dim,
                   d_idx, k_weight, index_k_weight, eps, rope, index_rope, k_cache, v_cache, index_k_cache, stream);
}

extern "C" int msa_latent_append(const void* latent, int64_t latent_stride, const void* k_rope, int64_t k_rope_stride,
                                 const msa_seqs* seqs, int latent_dim, const float* weight, float eps, const msa_rope* rope,
                                 void* cache, hipStream_t stream) {
  return latent_append(latent, latent_stride, k_rope, k_rope_stride, false, 1.f, seqs, latent_dim, weight, eps, rope, cache,
                       stream);
}

extern "C" int msa_latent_append_fp8(const void* latent, int64_t latent_stride, const void* k_rope, int64_t k_rope_stride,
                                     float cache_scale, const msa_seqs* seqs, int latent_dim, const float* weight, float eps,
                                     const msa_rope* rope, void* cache, hipStream_t stream) {
  return latent_append(latent, latent_stride, k_rope, k_rope_stride, true, cache_scale, seqs, latent_dim, weight, eps, rope,
                       cache, stream);
}
