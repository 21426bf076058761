// Latent attention, expanded form, on gfx950: causal attention with a key part
// of 128 elements and values of 128 per head, and a rotated key part of 64 that
// all heads share.
//
//   S_ij = scale (q_i . k_j + e_i . r_j),  O_i = sum_j softmax(S_i)_j v_j
//
// A CTA owns one head and a tile of consecutive query rows of one sequence, 32
// per wave, and streams the sequence's keys, 64 at a time, through a
// double-buffered LDS ring one sub-block ahead (copies without registers, issued
// between the score products).  A key's own part and values lie side by side in
// memory, the shared part apart from them; in LDS each has an area of its own, in
// the segment order that keeps its reads free of bank conflicts.  S^T = K Q^T is
// 12 products of 32x32x16 per 32 keys (8 own, 4 shared), O^T += V^T P^T 8; the
// online softmax of one sub-block runs between the value products of the one
// before, on fp32 scores, with running maximum and sum per row in registers.
//
// Few tiles: the steps (64 keys of a tile) of a head's tiles are dealt out evenly
// over the chip (latent_steps.h), shared tiles leave their parts in fp32, and
// latent_join_kernel joins them by the log-sum-exp rule in key order.
//
// Bound: matrix products.  8192 rows of 64 heads take 1226 - 1290 us, 1.1 PFLOP/s (1145 us at
// the rate of a large product); 2 x 512 rows on 14K - 16K keys 602 - 720 by the card (556).
#include <initializer_list>
#include <type_traits>

#include "flash_tile.h"
#include "latent_steps.h"

namespace {

using namespace msa;
using flash::copy16;
using flash::k_seg;
using flash::kAhead;
using flash::kDim;
using flash::kLn_2;
using flash::kLog2E;
using flash::lds_address;
using flash::lds_tr4;
using flash::v_seg;
using flash::xor32f;
using steps::kKeys;
using steps::Share;
using steps::TileGeom;
using steps::tile_geom;

constexpr int kRot = 64;                 // elements of the shared key part
constexpr int kPair = 2 * kDim;          // a key's own part and its values
constexpr float kSlack = 8.f;
// Steps per share, where there are few.  2 x 100 rows of 8 heads on 3000 keys, kernel and join in a graph: 24.9 us with
// 2, 24.3 with 4, 26.1 with 8.
constexpr int kMinSteps = 4;
constexpr int kHeld = 256;               // CTAs of 8 waves that the chip holds

struct ExpandedPlan {
  flash::Grid gr;                        // tiles of the unsplit grid
  int ranges;                            // shares per head; 0: a CTA per tile and head
  int min_steps;
};
struct ExpandedParts {
  float* o;                              // [CTA][2][rows x 128, in the accumulators' order], normalised
  float* lse;                            // [CTA][2][rows], base 2
  int4* tile;                            // [CTA]: the tile in slot 1: first query row, rows, parts (0: none)
};

// Segment s of row r of the shared part: rows are 128 bytes, half of the banks.
__device__ __forceinline__ int r_seg(int r, int s) { return s ^ ((r >> 1) & 7); }

template <int WAVES>
__global__ __launch_bounds__(WAVES* kWave, 2) void latent_attn_kernel(
    const uint16_t* __restrict__ q, int64_t q_stride, int64_t q_head, const uint16_t* __restrict__ e, int64_t e_stride,
    int64_t e_head, const uint16_t* __restrict__ kv, const uint16_t* __restrict__ kr, int64_t kr_stride, msa_seqs sq,
    ExpandedPlan pl, ExpandedParts parts, int H, float scale_log2, uint32_t q_flip, uint16_t* __restrict__ o,
    float* __restrict__ lse) {
  constexpr int kTile = 32 * WAVES;
  constexpr int KS = (kDim + kRot) / 16, KO = kDim / 16;     // k-steps of the scores, and of a key's own part
  constexpr int MT = kKeys / 32;
  constexpr int NK = 16 / WAVES, NR = 8 / WAVES;             // copies of 1 KiB per wave: own part (and values), shared part
  static_assert(WAVES <= 8, "");
  struct Ring {
    uint16_t k[2][kKeys * kDim], v[2][kKeys * kDim], r[2][kKeys * kRot];
  };
  __shared__ __align__(16) Ring ring;
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int n = lane & 31, h = lane >> 5;
  const int hd = static_cast<int>(blockIdx.x % H), which = static_cast<int>(blockIdx.x / H);

  // copies: lane l's 16 bytes land at 16 l of the wave's KiB, so it takes the segment that the row's order puts there
  const uint32_t kv_row = static_cast<uint32_t>(H * kPair * 2), r_row = static_cast<uint32_t>(kr_stride * 2);
  auto k_row = [&](int c) { return 4 * (c * WAVES + wave) + (lane >> 4); };
  auto s_row = [&](int c) { return 8 * (c * WAVES + wave) + (lane >> 3); };
  uint32_t koff[NK], voff[NK], roff[NR];
  // offsets of a sub-block's pieces; keys past row `last` repeat it: their values are finite, their weight zero
  auto hold_k = [&](int last) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NK; ++c) koff[c] = min(k_row(c), last) * kv_row + 16 * k_seg(k_row(c), lane & 15);
#pragma unroll
    for (int c = 0; c < NR; ++c) roff[c] = min(s_row(c), last) * r_row + 16 * r_seg(s_row(c), lane & 7);
  };
  auto hold_v = [&](int last) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NK; ++c) voff[c] = min(k_row(c), last) * kv_row + 2 * kDim + 16 * v_seg(k_row(c), lane & 15);
  };
  const uint32_t lds_k = lds_address(ring.k[0]), lds_v = lds_address(ring.v[0]), lds_r = lds_address(ring.r[0]);
  // MFMA operand reads, relative to a buffer
  uint32_t ks_at[KO], rs_at[KS - KO], vs_at[kDim / 32];
#pragma unroll
  for (int st = 0; st < KO; ++st) ks_at[st] = 2 * (n * kDim + 8 * k_seg(n, 2 * st + h));
#pragma unroll
  for (int st = 0; st < KS - KO; ++st) rs_at[st] = 2 * (n * kRot + 8 * r_seg(n, 2 * st + h));
  {
    // V^T operand: in each 16-lane group, lane j addresses row k0 + j/4, dims
    // n0 + 4(j%4) .. +3 of V and receives rows k0 .. k0+3 of dim n0 + j
    const int gq = lane >> 4, jj = lane & 15;
    const int rl = 4 * h + (jj >> 2);
#pragma unroll
    for (int td = 0; td < kDim / 32; ++td) {
      const int col = 32 * td + 16 * (gq & 1) + 4 * (jj & 3);
      vs_at[td] = 2 * (rl * kDim + 8 * v_seg(rl, col >> 3) + (col & 7));
    }
  }

  auto tile_rows = [&](const TileGeom& g, int s, int x, int64_t c_begin, int64_t c_end, auto describe) {
    const int t0 = x * kTile;
    const int t_end = min(t0 + kTile, g.q_rows);
    if (t_end <= t0) return;
    const int base_p = g.kv_len - g.q_rows;       // position of the sequence's first row
    const int seen = min(max(base_p + t_end, 0), g.kv_len);
    const int visits = (seen + kKeys - 1) / kKeys;
    const int b_begin = static_cast<int>(min<int64_t>(c_begin, visits)), b_end = static_cast<int>(min<int64_t>(c_end, visits));
    const int t = t0 + 32 * wave + n;
    const bool valid = t < t_end;
    const int p = valid ? base_p + t : -1;
    const bool live = t0 + 32 * wave < t_end;     // the wave has rows
    // sub-blocks below nfree are visible to every row of the wave and need no mask
    const int nfree = max(0, base_p + min(t0 + 32 * wave, t_end - 1) + 1) / kKeys;
    const int64_t row = static_cast<int64_t>(g.q_begin) + (valid ? t : t0);

    f32x16 acc_o[kDim / 32];
#pragma unroll
    for (int i = 0; i < kDim / 32; ++i) acc_o[i] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;
    // P of the pending sub-block in bf16, as the B operand of O^T = V^T P^T:
    // k-step u covers keys 16u + {4h + e, 8 + 4h + e}, e = 0..3
    bf16x8 bp[kKeys / 16];
    float alpha_pend = 1.f;                       // alpha of the sub-block whose P is in bp

    if (b_begin < b_end) {
      const int64_t first = seq_geom(sq, s).kv_start;
      const char* kb = reinterpret_cast<const char*>(kv + (first * H + hd) * kPair);
      const char* rb = reinterpret_cast<const char*>(kr + first * kr_stride);
      // The offsets are formed again for the sequence's last sub-block alone, where it is not full.
      hold_k(kKeys - 1);
      hold_v(kKeys - 1);
      auto copy_k = [&](int b, int buf) __attribute__((always_inline)) {
        const char* src = kb + static_cast<int64_t>(b) * kKeys * kv_row;
        const char* rsrc = rb + static_cast<int64_t>(b) * kKeys * r_row;
        const int last = g.kv_len - 1 - b * kKeys;
        if (last < kKeys - 1) hold_k(last);
#pragma unroll
        for (int c = 0; c < NK; ++c) copy16(src, koff[c], lds_k + buf * 2 * kKeys * kDim + 1024 * (c * WAVES + wave));
#pragma unroll
        for (int c = 0; c < NR; ++c) copy16(rsrc, roff[c], lds_r + buf * 2 * kKeys * kRot + 1024 * (c * WAVES + wave));
      };
      auto copy_v = [&](int b, int buf) __attribute__((always_inline)) {
        const char* src = kb + static_cast<int64_t>(b) * kKeys * kv_row;
        const int last = g.kv_len - 1 - b * kKeys;
        if (last < kKeys - 1) hold_v(last);
#pragma unroll
        for (int c = 0; c < NK; ++c) copy16(src, voff[c], lds_v + buf * 2 * kKeys * kDim + 1024 * (c * WAVES + wave));
      };
      bf16x8 bq[KS];                              // the query rows, as the B operand of S^T

      // S^T = K Q^T on one sub-block: lane (n, h) gets keys 32i + 8(a/4) + 4h + a%4 of row n.  Slots fenced off from one
      // another so that the compiler keeps the order; LDS operands are read kAhead slots ahead.
      auto scores = [&](int buf, f32x16 (&acc_s)[MT], auto beside) {
        const char* k0 = reinterpret_cast<const char*>(ring.k[buf]);
        const char* r0 = reinterpret_cast<const char*>(ring.r[buf]);
#pragma unroll
        for (int i = 0; i < MT; ++i) acc_s[i] = f32x16{};
        constexpr int NS = MT * KS;
        auto kread = [&](int j) -> bf16x8 {
          const int st = j % KS, i = j / KS;
          return ld_bf16x8(reinterpret_cast<const uint16_t*>(st < KO ? k0 + ks_at[st < KO ? st : 0] + 2 * 32 * i * kDim
                                                                     : r0 + rs_at[st < KO ? 0 : st - KO] + 2 * 32 * i * kRot));
        };
        bf16x8 kk[NS];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) kk[j] = kread(j);
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          if (j + kAhead < NS) kk[j + kAhead] = kread(j + kAhead);
          acc_s[j / KS] = mfma32x32x16(kk[j], bq[j % KS], acc_s[j / KS]);
          beside(j);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      auto mask = [&](f32x16 (&acc_s)[MT], int key0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int a = 0; a < 16; ++a) {
            const int key = key0 + 32 * i + 8 * (a >> 2) + 4 * h + (a & 3);
            acc_s[i][a] = key <= p ? acc_s[i][a] : -INFINITY;
          }
      };
      // eight weights as a B operand; their sum in fp32, as they are
      auto pack8 = [&](const f32x16& a, int e0, float& lsum) -> bf16x8 {
#pragma unroll
        for (int i = 0; i < 8; ++i) lsum += a[e0 + i];
        uint4 w;
        w.x = pack_bf16x2(a[e0 + 0], a[e0 + 1]);
        w.y = pack_bf16x2(a[e0 + 2], a[e0 + 3]);
        w.z = pack_bf16x2(a[e0 + 4], a[e0 + 5]);
        w.w = pack_bf16x2(a[e0 + 6], a[e0 + 7]);
        return __builtin_bit_cast(bf16x8, w);
      };
      // O is rescaled by the pending sub-block's alpha only when some row's maximum moved
      auto rescale = [&]() {
        if (__ballot(alpha_pend != 1.f)) {
#pragma unroll
          for (int i = 0; i < kDim / 32; ++i) acc_o[i] *= alpha_pend;
        }
      };
      // O^T += V^T P^T from one value sub-block in 16 fenced slots, beside(j) after the j-th
      auto pv = [&](int buf, auto beside) {
        constexpr int ND = kDim / 32, NO = (kKeys / 16) * ND;
        auto vread = [&](int j) {
          const char* a0 = reinterpret_cast<const char*>(ring.v[buf]) + vs_at[j % ND] + 2 * 16 * (j / ND) * kDim;
          const uint2 x0 = lds_tr4(reinterpret_cast<const uint16_t*>(a0));
          const uint2 x1 = lds_tr4(reinterpret_cast<const uint16_t*>(a0 + 2 * 8 * kDim));   // rows +8: same order
          return __builtin_bit_cast(bf16x8, make_uint4(x0.x, x0.y, x1.x, x1.y));
        };
        bf16x8 vr[NO];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) vr[j] = vread(j);
#pragma unroll
        for (int j = 0; j < NO; ++j) {
          if (j + kAhead < NO) vr[j + kAhead] = vread(j + kAhead);
          acc_o[j % ND] = mfma32x32x16(vr[j], bp[j / ND], acc_o[j % ND]);
          beside(j);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      // One sixteenth of a sub-block's softmax (raw scores; scale_log2 > 0 keeps their order): j = 0, 1 the maximum,
      // 2 .. 13 the weights, 14, 15 their sum and the packing.
      struct Soft {
        float m0, m_new, alpha, neg, lsum;
        bf16x8 bp[kKeys / 16];
      };
      auto soft_step = [&](Soft& z, f32x16 (&acc_s)[MT], int j) __attribute__((always_inline)) {
        if (j == 0) {
          z.m0 = -INFINITY;
          z.lsum = 0.f;
#pragma unroll
          for (int a = 0; a < 16; ++a) z.m0 = fmaxf(z.m0, acc_s[0][a]);
        } else if (j == 1) {
#pragma unroll
          for (int a = 0; a < 16; ++a) z.m0 = fmaxf(z.m0, acc_s[1][a]);
          z.m0 = fmaxf(z.m0, xor32f(z.m0));
          // the maximum that weights are relative to moves only when it is outgrown by 2^kSlack (else O would be
          // rescaled whenever some row's true one moves); the first visible keys outgrow -inf
          const bool grown = (z.m0 - m_run) * scale_log2 > kSlack;
          z.m_new = grown ? z.m0 : m_run;
          z.alpha = grown ? exp2_hw((m_run - z.m0) * scale_log2) : 1.f;
          z.neg = z.m_new == -INFINITY ? 0.f : -z.m_new * scale_log2;    // rows with nothing visible yet
        } else if (j < 14) {
#pragma unroll
          for (int x = 0; x < 32; ++x) {
            if (2 + (3 * x) / 8 != j) continue;
            acc_s[x >> 4][x & 15] = exp2_hw(fmaf(acc_s[x >> 4][x & 15], scale_log2, z.neg));
          }
        } else {
#pragma unroll
          for (int w = 2 * (j - 14); w < 2 * (j - 14) + 2; ++w) z.bp[w] = pack8(acc_s[w >> 1], 8 * (w & 1), z.lsum);
          if (j == 15) {
            z.lsum += xor32f(z.lsum);
            l_run = l_run * z.alpha + z.lsum;
            m_run = z.m_new;
          }
        }
      };
      auto take = [&](const Soft& z) {
#pragma unroll
        for (int w = 0; w < kKeys / 16; ++w) bp[w] = z.bp[w];
        alpha_pend = z.alpha;
      };
      // iteration b: K_{b+1} is in k[(b+1)&1], V_b in v[b&1]; after the S^T slots each O^T slot carries one sixteenth of
      // the next softmax, so the VALU works while the MFMA pipe drains.
      auto step = [&](int b, auto masked_t) {
        constexpr bool masked = decltype(masked_t)::value;
        __builtin_amdgcn_s_waitcnt(0);            // this thread's copies of K_{b+1} and V_b have landed
        __syncthreads();                          // everyone's have, and block b-1's readers are done
        auto move_k = [&]() __attribute__((always_inline)) {
          if (b + 2 < b_end) copy_k(b + 2, b & 1);
        };
        if (!live) {
          move_k();
          copy_v(b + 1, (b + 1) & 1);
          return;
        }
        rescale();
        __builtin_amdgcn_sched_barrier(0);
        f32x16 acc_s[MT];
        scores((b + 1) & 1, acc_s, [&](int j) __attribute__((always_inline)) {
          if (j == 18) move_k();
          if (j == 21) copy_v(b + 1, (b + 1) & 1);
        });
        Soft z;
        pv(b & 1, [&](int j) __attribute__((always_inline)) {
          if (masked && j == 0) mask(acc_s, (b + 1) * kKeys);
          soft_step(z, acc_s, j);
        });
        take(z);
      };

      // K and V of the first sub-block, K of the second
      copy_k(b_begin, b_begin & 1);
      copy_v(b_begin, b_begin & 1);
      if (b_begin + 1 < b_end) copy_k(b_begin + 1, (b_begin + 1) & 1);
      {
        const uint16_t* qp = q + row * q_stride + hd * q_head + 8 * h;
        const uint16_t* ep = e + row * e_stride + hd * e_head + 8 * h;
        u32x4 rq[KS];
#pragma unroll
        for (int st = 0; st < KS; ++st) rq[st] = valid ? load_raw(st < KO ? qp + 16 * st : ep + 16 * (st - KO)) : u32x4{};
#pragma unroll
        for (int st = 0; st < KS; ++st) bq[st] = __builtin_bit_cast(bf16x8, rq[st] ^ q_flip);
      }
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      if (live) {
        f32x16 acc_s[MT];
        scores(b_begin & 1, acc_s, [](int) {});
        if (b_begin >= nfree) mask(acc_s, b_begin * kKeys);
        Soft z;
#pragma unroll
        for (int j = 0; j < 16; ++j) soft_step(z, acc_s, j);
        take(z);
      }
      int b = b_begin;
      for (; b + 1 < min(nfree, b_end); ++b) step(b, std::false_type{});
      for (; b + 1 < b_end; ++b) step(b, std::true_type{});
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      if (live) {
        rescale();
        pv(b & 1, [](int) {});
      }
      __syncthreads();                            // the ring is free again
    }
    const bool whole = c_begin == 0 && b_end == visits;
    if (!whole && b_begin == 0 && b_begin < b_end) describe(visits);
    if (!valid) return;
    const bool empty = !(l_run > 0.f);
    const float inv_l = empty ? 0.f : 1.f / l_run;
    const float lse2 = empty ? -INFINITY : m_run * scale_log2 + __log2f(l_run);
    // O^T tile td: lane (n, h) holds d = 32td + 8(a/4) + 4h + a%4 of row n
    if (whole) {
      const int64_t head_row = row * H + hd;
      uint16_t* orow = o + head_row * kDim + 4 * h;
#pragma unroll
      for (int td = 0; td < kDim / 32; ++td)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          uint2 w;
          w.x = pack_bf16x2(acc_o[td][4 * e4 + 0] * inv_l, acc_o[td][4 * e4 + 1] * inv_l);
          w.y = pack_bf16x2(acc_o[td][4 * e4 + 2] * inv_l, acc_o[td][4 * e4 + 3] * inv_l);
          *reinterpret_cast<uint2*>(orow + 32 * td + 8 * e4) = w;
        }
      if (h == 0) lse[head_row] = lse2 * kLn_2;
    } else if (b_begin < b_end) {
      const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (b_begin > 0 ? 0 : 1);
      f32x4* po = reinterpret_cast<f32x4*>(parts.o + slot * kTile * kDim) + wave * 16 * kWave + lane;
#pragma unroll
      for (int td = 0; td < kDim / 32; ++td)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
          po[(td * 4 + e4) * kWave] =
              f32x4{acc_o[td][4 * e4], acc_o[td][4 * e4 + 1], acc_o[td][4 * e4 + 2], acc_o[td][4 * e4 + 3]} * inv_l;
      if (h == 0) parts.lse[slot * kTile + 32 * wave + n] = lse2;
    }
  };

  if (pl.ranges == 0) {
    int s, tile;
    flash::locate_tile(sq, pl.gr, which, kTile, &s, &tile);
    tile_rows(tile_geom(sq, s), s, tile, 0, INT32_MAX, [](int) {});
    return;
  }
  Share sh(sq, kTile, pl.ranges, pl.min_steps, which);
  if (threadIdx.x == 0) parts.tile[blockIdx.x] = make_int4(0, 0, 0, 0);
#pragma unroll 1
  for (; sh.more(); sh.next())
    tile_rows(sh.g, sh.s, sh.x, sh.begin(), sh.end(), [&](int visits) {
      if (threadIdx.x == 0)
        parts.tile[blockIdx.x] = make_int4(sh.g.q_begin + sh.x * kTile, min(kTile, sh.g.q_rows - sh.x * kTile), sh.parts(visits), 0);
    });
}

// Joins the parts of a tile that several shares had: a = max LSE_c,
// LSE = a + log sum 2^(LSE_c - a), O = sum 2^(LSE_c - LSE) O_c, in key order.  A CTA
// forms the list of such tiles; a wave takes a piece, 4 dimensions of 32 rows in
// each half of it.
constexpr int kJoinCtas = 1024;
__global__ __launch_bounds__(256) void latent_join_kernel(ExpandedParts parts, int ctas, int H, uint16_t* __restrict__ o,
                                                          float* __restrict__ lse) {
  constexpr int kTile = 256, kPieces = kTile * kDim / 4 / kWave, kWaves = 4;
  __shared__ int16_t list[kHeld];
  __shared__ int count[kWaves];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const bool has = static_cast<int>(threadIdx.x) < ctas && parts.tile[threadIdx.x].z > 0;    // ctas <= kHeld
  const uint64_t mask = __ballot(has);
  if (lane == 0) count[wave] = __popcll(mask);
  __syncthreads();
  int before = 0, tiles = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += count[w];
    tiles += count[w];
  }
  if (has) list[before + __popcll(mask & ((1ull << lane) - 1))] = static_cast<int16_t>(threadIdx.x);
  __syncthreads();
  for (int i = blockIdx.x * kWaves + wave; i < tiles * kPieces; i += gridDim.x * kWaves) {
    const int cta = list[i / kPieces], piece = i % kPieces;
    const int4 what = parts.tile[cta];
    const int np = what.z;
    const int e4 = piece & 3, td = (piece >> 2) & 3, r = 32 * (piece >> 4) + (lane & 31);
    if (r >= what.y) continue;             // rows behind the tile's have no parts
    constexpr int kBatch = 8;
    float top = -INFINITY, sum = 0.f;
    f32x4 y{};
    for (int c0 = 0; c0 < np; c0 += kBatch) {
      float l[kBatch];
      f32x4 v[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int c = c0 + b;
        l[b] = -INFINITY;
        v[b] = f32x4{};
        if (c < np) {
          const int64_t at = 2 * (cta + static_cast<int64_t>(c) * H) + (c == 0 ? 1 : 0);
          l[b] = parts.lse[at * kTile + r];
          v[b] = reinterpret_cast<const f32x4*>(parts.o + at * kTile * kDim)[piece * kWave + lane];
        }
      }
      float m = top;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) m = fmaxf(m, l[b]);
      const float base = m > -INFINITY ? m : 0.f;          // every part empty: all weights are zero
      const float f = exp2_hw(top - base);
      top = m;
      sum *= f;
      y *= f;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const float w = exp2_hw(l[b] - base);
        sum += w;
        y += v[b] * w;
      }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int64_t head_row = (static_cast<int64_t>(what.x) + r) * H + cta % H;
    uint2 w;
    w.x = pack_bf16x2(y[0] * inv, y[1] * inv);
    w.y = pack_bf16x2(y[2] * inv, y[3] * inv);
    *reinterpret_cast<uint2*>(o + head_row * kDim + 32 * td + 8 * e4 + 4 * (lane >> 5)) = w;
    if (td == 0 && e4 == 0 && lane < 32) lse[head_row] = sum > 0.f ? (top + __log2f(sum)) * kLn_2 : -INFINITY;
  }
}

// ---------------------------------------------------------------- host side
int validate_expanded(const msa_seqs* seqs, int H) {
  int st = msa_host::validate_seqs(seqs);
  if (st != MSA_OK) return st;
  if (H < 1) return MSA_ERR_INVALID;
  if (seqs->block_table) return MSA_ERR_UNSUPPORTED;   // contiguous key side only
  if (H > 256) return MSA_ERR_UNSUPPORTED;
  if (seqs->total_q_rows * H >= (int64_t(1) << 31)) return MSA_ERR_UNSUPPORTED;
  return MSA_OK;
}

// Waves per CTA (one CTA of 8 per CU, or two of 4), and whether the steps are
// dealt out or each tile has a CTA: what takes least by the sizes.  A step of a
// full tile of 8 waves takes 2.66 us, of 4 waves 1.25 alone on a CU and 2.8 with
// another beside it; shares cost 7 % more a step and 18 us for their ends, parts and join.  Tiles
// of a prompt see half of its keys on average, those of a chunk far behind a
// context all, so they end in rounds.  (The lengths are on the device; the key
// side's rows tell their mean where sequences lie one behind another.)
// Measured, us, 8 waves / 4 waves / shares: one prompt of 777 rows, 20 heads 32.9 /
// 23.5 / 30.9, 2000, 32 heads 73 / 61 / 88, 8000, 8 heads 236 / 200 / 211, 8192, 64
// heads 1282 / 1296 / 1380; 20 documents of 100 - 1000 rows, 32 heads 81 / 66 / 113;
// 2 x 512 rows on 16K keys, 64 heads 666 / 698 / 709, on 14 - 16K (another card) 720 /
// - / 756; 2 x 500 on 8K, 20 heads 245 / 183 / 125; 64 on 12K, 8 heads 207 / 226 / 33.
// Beyond 128 heads a head would have one share, which splits nothing and runs its tiles one behind another: 8 x 32
// rows on 2K, 129 heads 251 / 220 / 352, 3 x 256 on 16K, 136 heads 1132 / 1265 / 1354.  Where the heads do not divide 256
// fewer CTAs run, each faster for it, so the cost stays one of the whole chip: 2 x 200 on 8K, 100 heads (200
// CTAs) 265 / 304 / 267, of which 299 / 272 / 241 are told here, and 303 for the shares' CTAs counted.
constexpr double kShareStep = 1.07;
ExpandedPlan plan_of(const msa_seqs* seqs, int H, int* waves, int64_t* ctas) {
  const double rows = seqs->max_q_rows, keys = seqs->max_kv_len, seq_count = seqs->num_seqs;
  const bool chunk = 2 * rows <= keys;
  const double steps = std::max(1.0, keys / kKeys), avg = std::max(1.0, (keys - rows / 2) / kKeys);
  const double mean = std::min(1.0, seqs->total_kv_rows / (seq_count * std::max(1.0, keys)));
  auto tiles_with_rows = [&](int w) {      // at most
    const int64_t per_seq = (seqs->max_q_rows + 32 * w - 1) / (32 * w);
    return static_cast<double>(std::min<int64_t>(seqs->total_q_rows / (32 * w) + seqs->num_seqs, per_seq * seqs->num_seqs)) * H;
  };
  const double u8 = tiles_with_rows(8), u4 = tiles_with_rows(4);
  const double t8 = 2.66 * std::max(0.45, std::min(8.0, std::ceil(rows / 32)) / 8), t4 = 1.25, pair4 = 2.8;
  double whole8 = steps * t8, whole4 = steps * t4;
  if (chunk) {
    whole8 *= std::ceil(u8 / kHeld);
    if (u4 > 2 * kHeld) whole4 = std::ceil(u4 / (2 * kHeld)) * steps * pair4;
    else if (u4 > kHeld) whole4 = steps * (t4 + (u4 / kHeld - 1) * (pair4 - t4));
  } else {
    whole8 = std::max(whole8, u8 / kHeld * avg * t8 * mean);
    whole4 = std::max(whole4, u4 / (2 * kHeld) * avg * pair4 * mean);
  }
  // (shares have the last tiles' live waves alone to pay for)
  const double filled = std::min(u8, (seqs->total_q_rows / 32 + seq_count) / 8 * H);
  const double shares = filled / kHeld * avg * (rows >= 256 ? 2.66 : t8) * kShareStep * mean + 18;
  const int ranges = kHeld / H;            // shares per head
  ExpandedPlan pl{};
  *waves = 8;
  if (ranges > 1 && shares < std::min(whole8, whole4)) {
    pl.ranges = ranges;
    pl.min_steps = kMinSteps;
    *ctas = static_cast<int64_t>(pl.ranges) * H;
    return pl;
  }
  if (whole4 < whole8) *waves = 4;
  int64_t tiles;
  pl.gr = flash::plan_grid(seqs, 32 * *waves, seqs->max_q_rows, &tiles);
  *ctas = tiles * H;
  return pl;
}
size_t part_bytes(int64_t ctas, int waves) {
  return static_cast<size_t>(ctas) * (2 * 32 * waves * (kDim + 1) * sizeof(float) + sizeof(int4));
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

extern "C" size_t msa_latent_attn_workspace_size(const msa_seqs* seqs, int num_heads) {
  if (validate_expanded(seqs, num_heads) != MSA_OK) return 0;
  int waves;
  int64_t ctas;
  const ExpandedPlan pl = plan_of(seqs, num_heads, &waves, &ctas);
  return pl.ranges > 0 ? part_bytes(ctas, waves) : 0;
}

extern "C" int msa_latent_attn(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                               int64_t q_rope_stride, int64_t q_rope_head_stride, const void* kv, const void* k_rope,
                               int64_t k_rope_stride, const msa_seqs* seqs, int num_heads, float softmax_scale, void* o,
                               float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int st = validate_expanded(seqs, num_heads);
  if (st != MSA_OK) return st;
  if (seqs->total_q_rows == 0) return MSA_OK;
  if (!q || !q_rope || !o || !lse) return MSA_ERR_INVALID;
  if (seqs->total_kv_rows > 0 && (!kv || !k_rope)) return MSA_ERR_INVALID;
  if (q_stride < 0 || q_head_stride < 0 || q_rope_stride < 0 || q_rope_head_stride < 0 || k_rope_stride < 0)
    return MSA_ERR_INVALID;
  for (const void* x : {q, q_rope, kv, k_rope, static_cast<const void*>(o)})
    if (!aligned16(x)) return MSA_ERR_UNSUPPORTED;
  if ((q_stride | q_head_stride | q_rope_stride | q_rope_head_stride | k_rope_stride) % 8 != 0) return MSA_ERR_UNSUPPORTED;
  if (k_rope_stride > (int64_t(1) << 20)) return MSA_ERR_UNSUPPORTED;     // 64 rows' offsets are 32 bits
  int waves;
  int64_t ctas;
  const ExpandedPlan pl = plan_of(seqs, num_heads, &waves, &ctas);
  if (ctas * waves >= (int64_t(1) << 26)) return MSA_ERR_UNSUPPORTED;    // a grid's limit
  ExpandedParts parts{};
  if (pl.ranges > 0) {
    if (!workspace || workspace_bytes < part_bytes(ctas, waves)) return MSA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MSA_ERR_UNSUPPORTED;
    const int64_t rows = 2 * ctas * 32 * waves;
    parts.o = static_cast<float*>(workspace);
    parts.lse = parts.o + rows * kDim;
    parts.tile = reinterpret_cast<int4*>(parts.lse + rows);
  }
  const flash::LogitScale scale = flash::logit_scale(softmax_scale * kLog2E);
  auto run = [&](auto count) {
    constexpr int W = decltype(count)::value;
    msa_prof::launch(W == 8 ? "latent_attn_kernel" : "latent_attn_narrow_kernel", latent_attn_kernel<W>,
                     dim3(static_cast<unsigned>(ctas)), dim3(W * kWave), 0, stream,
                     static_cast<const uint16_t*>(q), q_stride, q_head_stride, static_cast<const uint16_t*>(q_rope),
                     q_rope_stride, q_rope_head_stride, static_cast<const uint16_t*>(kv), static_cast<const uint16_t*>(k_rope),
                     k_rope_stride, *seqs, pl, parts, num_heads, scale.log2, scale.q_flip, static_cast<uint16_t*>(o), lse);
  };
  if (waves == 4) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 8>{});
  if (pl.ranges > 0)
    msa_prof::launch("latent_join_kernel", latent_join_kernel, dim3(kJoinCtas), dim3(256), 0, stream, parts,
                     static_cast<int>(ctas), num_heads, static_cast<uint16_t*>(o), lse);
  return msa_host::launch_status();
}
