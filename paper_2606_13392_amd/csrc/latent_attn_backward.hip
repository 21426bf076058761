// Gradients of latent attention's expanded form on gfx950.
//
// With P_ij = exp(scale (q_i . k_j + e_i . r_j) - LSE_i), D_i = dO_i . O_i and
// dS_ij = P_ij (dO_i . v_j - D_i), for each head:
//   dq_i = scale sum_j dS_ij k_j,  de_i = scale sum_j dS_ij r_j,
//   dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dO_i,
// and summed over the heads  dr_j = scale sum_h sum_i dS_ij e_i.
//
// Two kernels of one form, so that every sum has an order of its own and no
// result depends on which CTA comes first: a wave keeps rows of one side as matrix
// operands in registers (64 or 32 queries and dO, or 32 keys and values), the CTA streams
// the other side 64 rows at a time through LDS, and a wave forms both score products
// and adds the weights' products with the streamed rows, read down their columns.
// What this repeats, the score products of the second kernel, is 20 of 72 matrix
// products per 32 x 32; adding the queries' gradients from the key side would take
// atomics, or a store and load of every dS (8192 rows of 64 heads: 9 GB, 1.7 ms at
// a copy's rate, against the 1.1 ms that the repeated products take).
//
// The products of one 32 streamed rows run ahead of the additions of the 32
// before, between which the weights are formed.  The shared part's gradient leaves
// per head in fp32 and latent_sum_kernel adds the heads in their order; it also
// clears what no sequence owns.
//
// P and dS are rounded to bf16 as operands of the additions, in the same way the
// forward rounds P; the sums are fp32 and leave in bf16, the shared part's after the
// heads' sum in fp32.
//
// Bound: issue.  A wave has its SIMD alone (its operands and sums are 350 - 500
// registers), and between two matrix products of 32 clocks it issues some five other
// instructions.  8192 rows of 64 heads: queries 1.83 - 1.89 ms, keys 2.60 - 2.70 (1.85 and 2.30 at the
// rate of a large matrix product, repeated products counted), the heads' sum 0.03.
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "flash_tile.h"
#include "latent_steps.h"

namespace {

using namespace msa;
using flash::copy16;
using flash::kDim;
using flash::kLog2E;
using flash::lds_address;
using flash::lds_tr4;
using flash::xor32f;
using steps::TileGeom;
using steps::tile_geom;

constexpr int kRot = 64;                 // elements of the shared key part
constexpr int kPair = 2 * kDim;          // a key's own part and its values
constexpr int kRowsT = 64;               // streamed rows per tile
constexpr int kRing = 3;
constexpr int kWaves = 4;                // one per SIMD: a wave's operands and sums take 240 (keys) or 352 registers
constexpr int kThreads = kWaves * kWave;
constexpr int kRowTile = 64 * kWaves, kKeyTile = 32 * kWaves;      // stationary rows per CTA

// Streamed rows in LDS: 16-byte segments, permuted by the row so that reads of
// 16 rows' segment and transposing reads of 4 rows x 4 segments fall on all
// banks: rows of 256 bytes and of 128 (odd ones start in the other half of the
// banks).  The permutations are XORs, so an operand's address is one XOR from
// another's.
__device__ __forceinline__ int wide_mix(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }
__device__ __forceinline__ int half_mix(int r) { return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3); }

typedef u32x4 u32x4_at8 __attribute__((aligned(8)));               // gradients of queries may stand at any multiple of 8

struct Tile {
  uint16_t own[kRowsT * kDim], other[kRowsT * kDim], rot[kRowsT * kRot];
};

// A streamed query's statistics as three bf16 each, the largest first, 24 bits
// together: -LSE / scale in x and y, -D in z and w.  As an operand of a matrix
// product against ones they start both scores' sums, in place of eight reads of four
// numbers each per 32 rows: the reads of LDS are what bounds the keys' kernel.
// kFar (of -scale's sign) takes every weight to 0; |scale| is at least kLeast, so that
// the quotient of a scale of 0 is a number (all below it is 0 to an exponent).
constexpr float kFar = 0x1p120f, kLeast = 0x1p-100f;
__device__ __forceinline__ uint2 three_bf16(float x) {
  const uint32_t hi = pack_bf16x2(x, 0.f) & 0xFFFFu;
  const float r = x - __uint_as_float(hi << 16);
  const uint32_t mid = pack_bf16x2(r, 0.f) & 0xFFFFu;
  return make_uint2(hi | mid << 16, pack_bf16x2(r - __uint_as_float(mid << 16), 0.f) & 0xFFFFu);
}

struct Side {                            // [rows, heads] vectors: elements between rows and between heads
  const uint16_t* p;
  int64_t row, head;
};
struct Grad {
  uint16_t* p;
  int64_t row, head;
};
struct Args {
  Side q, e, k, v, r, o, d_o;            // k, v: a key's own part and values; r: the shared part (head 0)
  const float* lse;                      // [T, H]
  Grad d_q, d_e, d_k, d_v;
  uint4* stat;                           // [H][T]
  float* d_r;                            // [H][total_kv][64], before the scale
  int H;
  float scale, scale_log2;
};

// KEYS: keys are stationary, 32 to a wave (NT = 1), and queries streamed; else queries are
// stationary, 32 NT to a wave, and keys streamed.  With 64 an operand read from LDS
// feeds two products (the keys' sums leave no registers for that), with 32 a tile takes
// little more than half the time and there are twice the CTAs.  Queries' kernel, 64 and 32 to a wave:
// 1 x 512 rows, 8 heads (16 CTAs of 256 rows) 35 and 22 us, 1 x 2048, 20 (160) 107 and 70, 1 x 4096,
// 16 (256) 226 and 171, 10 x 300, 20 (400) 60 and 48, documents of 300 - 3000 rows, 32 (928) 241 and 245.
constexpr int64_t kFewTiles = 768;
template <bool KEYS, int NT>
__global__ __launch_bounds__(kThreads, 1) void latent_backward_kernel(Args a, msa_seqs sq, flash::Grid gr) {
  constexpr int KO = kDim / 16, KS = (kDim + kRot) / 16;
  constexpr int ND = KS / 2;                       // 32-dimension tiles of own and shared part
  constexpr int NA = KEYS ? ND + kDim / 32 : ND;   // accumulator tiles
  constexpr bool kRoomy = NT == 1;                 // registers are left for addresses
  constexpr int kTileRows = 32 * NT * kWaves;
  constexpr int NK = 16 / kWaves, NR = 8 / kWaves; // copies of 1 KiB per wave: wide rows, half rows
  constexpr int kAhead = kRoomy ? 5 : 3;
  __shared__ __align__(16) Tile ring[kRing];
  __shared__ __align__(16) uint4 stat[kRing][KEYS ? kRowsT : 1];      // of streamed queries
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int n = lane & 31, h = lane >> 5;
  const int hd = static_cast<int>(blockIdx.x % a.H), which = static_cast<int>(blockIdx.x / a.H);

  // ------------------------------------------------ the CTA's tile of stationary rows
  int s = 0, tile = 0;
  if constexpr (KEYS) {
    // tiles are numbered through, sequence after sequence; a lane counts four sequences', whose loads are under way
    // together (4000 sequences of 10 rows, 8 heads: 2.06 ms, with one a lane 3.17)
    constexpr int kPer = 4;
    int base = 0;
    bool found = false;
    for (int c = 0; c < sq.num_seqs && !found; c += kPer * kWave) {
      int mine[kPer], sum = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int x = c + kPer * lane + i;
        mine[i] = (max(tile_geom(sq, min(x, sq.num_seqs - 1)).kv_len, 0) + kKeyTile - 1) / kKeyTile;
        mine[i] = x < sq.num_seqs ? mine[i] : 0;
        sum += mine[i];
      }
      int incl = sum;
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const int x = __shfl_up(incl, d);
        if (lane >= d) incl += x;
      }
      const int all = __builtin_amdgcn_readlane(incl, kWave - 1);
      if (which < base + all) {
        const int j = __popcll(__ballot(which >= base + incl));
        tile = which - base - (j > 0 ? __builtin_amdgcn_readlane(incl, j - 1) : 0);
        s = c + kPer * j;
#pragma unroll
        for (int i = 0; i + 1 < kPer; ++i) {
          const int x = __builtin_amdgcn_readlane(mine[i], j);
          if (tile < x) break;
          tile -= x;
          ++s;
        }
        found = true;
      }
      base += all;
    }
    if (!found) return;
  } else {
    flash::locate_tile(sq, gr, which, kTileRows, &s, &tile);
  }
  const TileGeom g = tile_geom(sq, s);
  const int64_t first_key = seq_geom(sq, s).kv_start;
  const int base_p = g.kv_len - g.q_rows;          // position of the sequence's first query row
  const int limit = KEYS ? g.kv_len : g.q_rows;
  const int x0 = tile * kTileRows;                 // first stationary row
  if (x0 >= limit) return;
  const int x_end = min(x0 + kTileRows, limit);
  const int w0 = x0 + 32 * NT * wave;              // the wave's first; the lane's are w0 + n + 32 nt
  const int64_t base_x = KEYS ? first_key : g.q_begin;
  const int streamed = KEYS ? g.q_rows : g.kv_len; // rows of the other side
  // tiles of streamed rows that some stationary row meets
  const int first_row = KEYS ? max(0, x0 - base_p) : 0;
  const int end_row = KEYS ? g.q_rows : min(max(base_p + x_end, 0), g.kv_len);
  const int b_begin = first_row / kRowsT, b_end = first_row < end_row ? (end_row + kRowsT - 1) / kRowsT : b_begin;

  // ------------------------------------------------ copies of streamed rows
  const Side own = KEYS ? a.q : a.k, other = KEYS ? a.d_o : a.v, rot = KEYS ? a.e : a.r;
  const int64_t row0 = KEYS ? g.q_begin : first_key;
  const char* own_p = reinterpret_cast<const char*>(own.p + row0 * own.row + hd * own.head);
  const char* other_p = reinterpret_cast<const char*>(other.p + row0 * other.row + hd * other.head);
  const char* rot_p = reinterpret_cast<const char*>(rot.p + row0 * rot.row + hd * rot.head);
  const uint32_t own_s = static_cast<uint32_t>(own.row * 2), other_s = static_cast<uint32_t>(other.row * 2),
                 rot_s = static_cast<uint32_t>(rot.row * 2);
  const uint32_t lds0 = lds_address(&ring[0]);
  constexpr uint32_t kOwnAt = 0, kOtherAt = sizeof(uint16_t) * kRowsT * kDim, kRotAt = 2 * kOtherAt;
  // a tile's copies, one at a time: piece 0 .. 2 NK - 1 wide rows, then half rows, then (KEYS) the statistics
  constexpr int kCopies = 2 * NK + NR;
  struct From {
    const char *own, *other, *rot, *stat;
    int last;                                      // rows past the end repeat the last one
    uint32_t dst, dst_stat;
  };
  auto source = [&](int b, int buf) {
    const int64_t at = static_cast<int64_t>(b) * kRowsT;
    From f;
    f.own = own_p + at * own_s;
    f.other = other_p + at * other_s;
    f.rot = rot_p + at * rot_s;
    f.stat = reinterpret_cast<const char*>(a.stat + hd * sq.total_q_rows + row0 + at);
    f.last = streamed - 1 - b * kRowsT;
    f.dst = lds0 + buf * static_cast<uint32_t>(sizeof(Tile)) + 1024 * wave;
    f.dst_stat = lds_address(&stat[0][0]) + buf * static_cast<uint32_t>(sizeof(stat[0]));
    return f;
  };
  // Where registers are left a lane's offsets are held, and formed again for the last tile alone
  auto offset = [&](int c, int ln, int last) __attribute__((always_inline)) -> uint32_t {
    if (c < 2 * NK) {
      const int r = 4 * ((c >> 1) * kWaves + wave) + (ln >> 4);
      return min(r, last) * (c & 1 ? other_s : own_s) + 16 * ((ln & 15) ^ wide_mix(r));
    }
    const int r = 8 * ((c - 2 * NK) * kWaves + wave) + (ln >> 3);
    return c < kCopies ? min(r, last) * rot_s + 16 * ((ln & 7) ^ half_mix(r)) : 16 * min(ln, last);
  };
  constexpr int kAllCopies = kCopies + (KEYS ? 1 : 0);
  uint32_t held[kRoomy ? kAllCopies : 1];
  auto hold = [&](int last) __attribute__((always_inline)) {
    if constexpr (kRoomy)
#pragma unroll
      for (int c = 0; c < kAllCopies; ++c) {
        held[c] = offset(c, lane, last);
        asm volatile("" : "+v"(held[c]));
      }
  };
  auto copy_piece = [&](const From& f, int c, int ln) __attribute__((always_inline)) {
    const uint32_t at = kRoomy ? held[kRoomy ? c : 0] : offset(c, ln, f.last);
    if (c < 2 * NK) {
      if (c & 1) copy16(f.other, at, f.dst + kOtherAt + 1024 * kWaves * (c >> 1));
      else copy16(f.own, at, f.dst + kOwnAt + 1024 * kWaves * (c >> 1));
    } else if (c < kCopies) {
      copy16(f.rot, at, f.dst + kRotAt + 1024 * kWaves * (c - 2 * NK));
    } else {
      copy16(f.stat, at, f.dst_stat);              // each wave the same: the count is alike
    }
  };
  auto copy = [&](int b, int buf) {
    const From f = source(b, buf);
    int ln = lane;
    asm volatile("" : "+v"(ln));                   // offsets are formed here each time: held, they spill
    hold(f.last);
#pragma unroll
    for (int c = 0; c < kAllCopies; ++c) copy_piece(f, c, ln);
  };
  if (b_begin < b_end) {
    copy(b_begin, 0);
    if (b_begin + 1 < b_end) copy(b_begin + 1, 1);
  }

  // ------------------------------------------------ stationary operands
  bf16x8 b1[NT][KS], b2[NT][KO];
  float lane_lse[NT] = {}, lane_d[NT] = {};
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const Side f = KEYS ? a.k : a.q, t = KEYS ? a.r : a.e, w = KEYS ? a.v : a.d_o;
    const bool valid = w0 + 32 * nt + n < limit;
    const int64_t mine = base_x + (valid ? w0 + 32 * nt + n : x0);
    const uint16_t* fp = f.p + mine * f.row + hd * f.head + 8 * h;
    const uint16_t* tp = t.p + mine * t.row + hd * t.head + 8 * h;
    const uint16_t* wp = w.p + mine * w.row + hd * w.head + 8 * h;
#pragma unroll
    for (int st = 0; st < KS; ++st) b1[nt][st] = ld_bf16x8(st < KO ? fp + 16 * st : tp + 16 * (st - KO));
#pragma unroll
    for (int st = 0; st < KO; ++st) b2[nt][st] = ld_bf16x8(wp + 16 * st);
    if constexpr (!KEYS) {
      const uint16_t* op = a.o.p + mine * a.o.row + hd * a.o.head + 8 * h;
#pragma unroll
      for (int st = 0; st < KO; ++st) {
        const bf16x8 ov = ld_bf16x8(op + 16 * st);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          lane_d[nt] = fmaf(static_cast<float>(ov[i]), static_cast<float>(b2[nt][st][i]), lane_d[nt]);
      }
      lane_d[nt] += xor32f(lane_d[nt]);
      // a row that meets no key has an LSE of -infinity; +infinity keeps its weights 0 behind the mask too
      const float lse = a.lse[mine * a.H + hd];
      lane_lse[nt] = lse == -INFINITY ? INFINITY : lse * kLog2E;
      if (valid && h == 0) {
        const float far = copysignf(kFar, -a.scale_log2), x = lane_lse[nt] / -a.scale_log2;
        const uint2 l = three_bf16(lse == -INFINITY ? far : x > kFar ? kFar : x < -kFar ? -kFar : x), d = three_bf16(-lane_d[nt]);
        a.stat[hd * sq.total_q_rows + mine] = make_uint4(l.x, l.y, d.x, d.y);
      }
    }
  }

  // ------------------------------------------------ operand addresses
  // Where registers are left each is held, from the start of the ring; else formed from the first where they are read: no register is left
  constexpr int kWideAt = kRoomy ? KO : 1, kHalfAt = kRoomy ? kRot / 16 : 1;
  uint32_t row_own[kWideAt], row_rot[kHalfAt], col_own[kWideAt], col_rot[kHalfAt];
  {
    // transposed operand: in each 16-lane group, lane j addresses row k0 + j/4, dims n0 + 4(j%4) .. +3 and
    // receives rows k0 .. k0+3 of dim n0 + j
    const int gq = lane >> 4, jj = lane & 15;
    const int rl = 4 * h + (jj >> 2), seg = 2 * (gq & 1) + ((jj & 3) >> 1);
#pragma unroll
    for (int j = 0; j < kWideAt; ++j) {
      row_own[j] = n * 2 * kDim + 16 * (h ^ wide_mix(n)) ^ 32 * j;
      col_own[j] = (rl * 2 * kDim + 16 * (seg ^ wide_mix(rl)) + 8 * (jj & 1)) ^ 32 * j;
    }
#pragma unroll
    for (int j = 0; j < kHalfAt; ++j) {
      row_rot[j] = n * 2 * kRot + 16 * (h ^ half_mix(n)) ^ 32 * j;
      col_rot[j] = (rl * 2 * kRot + 16 * (seg ^ half_mix(rl)) + 8 * (jj & 1)) ^ (64 * (j >> 1) + 16 * (j & 1));
    }
  }
  // the rows', the columns' addresses on to another buffer, where they are held
  auto move = [&](uint32_t (&wide)[kWideAt], uint32_t (&half)[kHalfAt], int from, int to) __attribute__((always_inline)) {
    if constexpr (kRoomy) {
      const int by = (to - from) * static_cast<int>(sizeof(Tile));
#pragma unroll
      for (int j = 0; j < kWideAt; ++j) {
        wide[j] += by;
        asm volatile("" : "+v"(wide[j]));
      }
#pragma unroll
      for (int j = 0; j < kHalfAt; ++j) {
        half[j] += by;
        asm volatile("" : "+v"(half[j]));
      }
    }
  };
  auto tr8 = [](const char* p0, const char* p1) {
    const uint2 y0 = lds_tr4(reinterpret_cast<const uint16_t*>(p0)), y1 = lds_tr4(reinterpret_cast<const uint16_t*>(p1));
    return __builtin_bit_cast(bf16x8, make_uint4(y0.x, y0.y, y1.x, y1.y));
  };

  f32x16 acc[NA][NT];
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[i][nt] = f32x16{};
  bf16x8 ps[NT][2], pp[NT][2];                           // pending dS and (KEYS) P of 32 streamed rows, as B operands

  // a statistic's three parts are elements 0 .. 2 of the lanes h = 0
  const bf16x8 ones = __builtin_bit_cast(bf16x8, h == 0 ? make_uint4(0x3F803F80u, 0x3F80u, 0, 0) : make_uint4(0, 0, 0, 0));
  // (Roomy) Each phase reads the first kAhead operands of the next in its last slots, where these are there: the reads'
  // time is bare else.  (Of the queries' kernel, with products enough, it takes 3 % more time.)
  bf16x8 pre[kAhead];
  // operands of the products of rows 32 half .. + 31, and of the additions of those rows
  auto read_row = [&](int buf, int half, int j) __attribute__((always_inline)) -> bf16x8 {
    const char* t = reinterpret_cast<const char*>(&ring[kRoomy ? 0 : buf]);
    const int k = j < KS ? j : j - KS;             // 16 dimensions; KO .. KS - 1 of the shared part
    uint32_t at;
    if constexpr (kRoomy) {
      at = k < KO ? row_own[k < KO ? k : 0] : row_rot[k < KO ? 0 : k - KO];
    } else {
      at = (k < KO ? row_own[0] : row_rot[0]) ^ 32 * (k < KO ? k : k - KO);
    }
    t += k < KO ? (j < KS ? kOwnAt : kOtherAt) + half * 32 * 2 * kDim : kRotAt + half * 32 * 2 * kRot;
    return ld_bf16x8(reinterpret_cast<const uint16_t*>(t + at));
  };
  auto read_col = [&](int buf, int half, int j) __attribute__((always_inline)) -> bf16x8 {
    const char* t = reinterpret_cast<const char*>(&ring[kRoomy ? 0 : buf]);
    const int u = j / NA, i = j % NA;              // 16 streamed rows, accumulator tile
    const int r = 32 * half + 16 * u;
    const bool wide = i < KO / 2 || i >= ND;
    const int k = i < KO / 2 ? i : i < ND ? i - KO / 2 : i - ND;
    uint32_t at0, at1;
    if constexpr (kRoomy) {
      at0 = wide ? col_own[wide ? 2 * k : 0] : col_rot[wide ? 0 : 2 * k];
      at1 = wide ? col_own[wide ? 2 * k + 1 : 0] : col_rot[wide ? 0 : 2 * k + 1];
    } else {
      at0 = (wide ? col_own[0] : col_rot[0]) ^ 64 * k;
      at1 = at0 ^ (wide ? 32 : 16);
    }
    t += wide ? (i < ND ? kOwnAt : kOtherAt) + r * 2 * kDim : kRotAt + r * 2 * kRot;
    return tr8(t + at0, t + at1 + 8 * (wide ? 2 * kDim : 2 * kRot));
  };
  // both score products of streamed rows 32 half .. + 31: lane (n, h) gets rows 8(i/4) + 4h + i%4 against its own
  auto products = [&](int buf, int half, f32x16 (&z)[NT], f32x16 (&dz)[NT], auto beside) __attribute__((always_inline)) {
    if constexpr (!kRoomy) asm volatile("" : "+v"(row_own[0]), "+v"(row_rot[0]));    // as above
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) z[nt] = dz[nt] = f32x16{};
    if constexpr (KEYS) {
      const uint4 x = stat[buf][32 * half + n];
      z[0] = mfma32x32x16(__builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, 0, 0)), ones, z[0]);
      dz[0] = mfma32x32x16(__builtin_bit_cast(bf16x8, make_uint4(x.z, x.w, 0, 0)), ones, dz[0]);
    }
    bf16x8 op[KS + KO];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) op[j] = kRoomy ? pre[j] : read_row(buf, half, j);
#pragma unroll
    for (int j = 0; j < KS + KO; ++j) {
      if (j + kAhead < KS + KO) op[j + kAhead] = read_row(buf, half, j + kAhead);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (j < KS) z[nt] = mfma32x32x16(op[j], b1[nt][j < KS ? j : 0], z[nt]);
        else dz[nt] = mfma32x32x16(op[j], b2[nt][j < KS ? 0 : j - KS], dz[nt]);
      }
      beside(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // adds the pending weights' products with their streamed rows; beside(j) after the j-th slot
  constexpr int kSlots = 2 * NA;
  auto additions = [&](int buf, int half, auto beside) __attribute__((always_inline)) {
    if constexpr (!kRoomy) asm volatile("" : "+v"(col_own[0]), "+v"(col_rot[0]));    // as above
    bf16x8 op[kSlots];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) op[j] = kRoomy ? pre[j] : read_col(buf, half, j);
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
      if (j + kAhead < kSlots) op[j + kAhead] = read_col(buf, half, j + kAhead);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        acc[j % NA][nt] = mfma32x32x16(op[j], j % NA < ND ? ps[nt][j / NA] : pp[nt][j / NA], acc[j % NA][nt]);
      beside(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // P and dS of 32 streamed rows in kSlots pieces: z becomes P, dz dS.  The last two pieces pack them, each after the
  // last slot that adds what was there before.
  const float far = copysignf(kFar, a.scale_log2);
  const int edge = (KEYS ? w0 + n - base_p : base_p + w0 + n) - 4 * h;
  auto expo = [&](int row, auto masked, f32x16 (&z)[NT], int i) __attribute__((always_inline)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p = exp2_hw(KEYS ? z[nt][i] * a.scale_log2 : fmaf(z[nt][i], a.scale_log2, -lane_lse[nt]));
      if constexpr (!KEYS && decltype(masked)::value) {
        const int y = 8 * (i / 4) + i % 4;         // of the streamed row, less row + 4 h
        p = y <= edge + 32 * nt - row ? p : 0.f;
      }
      z[nt][i] = p;
    }
  };
  // Of the 16, this many go between the second score products, which need no result of theirs: additions of 24 matrix
  // products do not cover all the work on 32 x 64 weights (8K rows of one sequence: 1.90 ms; with none 1.96, with 16
  // the same), those of 20 cover the work on 32 x 32.
  constexpr int kEarly = KEYS ? 0 : 12;
  auto early = [&](int row, auto masked, f32x16 (&z)[NT], int j) __attribute__((always_inline)) {
    constexpr int kFirst = KS + 1, kMany = KO - 1;
#pragma unroll
    for (int i = 0; i < kEarly; ++i)
      if (j == kFirst + i * kMany / max(kEarly, 1)) expo(row, masked, z, i);
  };
  auto weigh = [&](int row, auto masked, f32x16 (&z)[NT], f32x16 (&dz)[NT], int j) __attribute__((always_inline)) {
    constexpr int kLast = kSlots - 2;
    static_assert(kLast >= NA, "");
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i * kLast / 16 != j) continue;
      if (i >= kEarly) expo(row, masked, z, i);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) dz[nt][i] = z[nt][i] * (KEYS ? dz[nt][i] : dz[nt][i] - lane_d[nt]);
    }
    if (j >= kLast) {
      const int u = j - kLast;
      auto pack = [&](const f32x16& v) {
        uint4 y;
        y.x = pack_bf16x2(v[8 * u + 0], v[8 * u + 1]);
        y.y = pack_bf16x2(v[8 * u + 2], v[8 * u + 3]);
        y.z = pack_bf16x2(v[8 * u + 4], v[8 * u + 5]);
        y.w = pack_bf16x2(v[8 * u + 6], v[8 * u + 7]);
        return __builtin_bit_cast(bf16x8, y);
      };
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        ps[nt][u] = pack(dz[nt]);
        if constexpr (KEYS) pp[nt][u] = pack(z[nt]);
      }
    }
  };
  // (queries) whether some lane of the wave does not meet some row of tile b
  auto is_masked = [&](int b) { return (b + 1) * kRowsT > base_p + w0 + 1; };
  // (KEYS) the scores of streamed rows, from row on, that a key does not meet; the branch is free, two loops spill
  auto mask = [&](int row, f32x16 (&z)[NT]) __attribute__((always_inline)) {
    if constexpr (!KEYS) return;
    if (base_p + row >= w0 + 31) return;
    const int first = edge - row;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[0][i] = 8 * (i / 4) + i % 4 >= first ? z[0][i] : -far;
    asm volatile("" : "+v"(z[0]));
  };
  auto sync = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  // tile b's copies, all waves'; queries past the end get no weight
  auto arrive = [&](int b, int buf) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (KEYS) {
      if ((b + 1) * kRowsT > streamed && b * kRowsT + lane >= streamed)
        stat[buf][lane] = make_uint4(a.scale_log2 < 0 ? 0x7B80u : 0xFB80u, 0, 0, 0);     // kFar, of -scale's sign
    }
    sync();
  };

  if (b_begin < b_end) {
    arrive(b_begin, 0);
    f32x16 z[NT], dz[NT];
    // the first operands of the products, of the additions that come next: behind slot j of j_end
    auto rows_next = [&](int buf, int half, int j, int j_end) __attribute__((always_inline)) {
      if (kRoomy && j >= j_end - kAhead) pre[j - (j_end - kAhead)] = read_row(buf, half, j - (j_end - kAhead));
    };
    auto cols_next = [&](int buf, int half, int j, int j_end) __attribute__((always_inline)) {
      if (kRoomy && j >= j_end - kAhead) pre[j - (j_end - kAhead)] = read_col(buf, half, j - (j_end - kAhead));
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) rows_next(0, 0, j, kAhead);
    products(0, 0, z, dz, [&](int j) __attribute__((always_inline)) {
      early(b_begin * kRowsT, std::true_type{}, z, j);
      rows_next(0, 1, j, KS + KO);
    });
    mask(b_begin * kRowsT, z);
#pragma unroll
    for (int j = 0; j < kSlots; ++j) weigh(b_begin * kRowsT, std::true_type{}, z, dz, j);
    // Rows 32 .. 63 of tile b, then rows 0 .. 31 of tile b + 1: the products of these, the additions of those before.
    // Behind the barrier tile b + 1 is there and tile b - 1's readers are done: its buffer takes tile b + 2,
    // whose copies go out between the products.  (Behind the last tiles they repeat the last one.)
    int b = b_begin, buf = 0;
    auto first = [&](auto masked) __attribute__((always_inline)) {
      products(buf, 1, z, dz, [&](int j) __attribute__((always_inline)) {
        early(b * kRowsT + 32, masked, z, j);
        cols_next(buf, 0, j, KS + KO);
      });
      mask(b * kRowsT + 32, z);
    };
    auto step = [&](auto masked) __attribute__((always_inline)) {
      const int next = buf == kRing - 1 ? 0 : buf + 1;
      first(masked);
      additions(buf, 0, [&](int j) __attribute__((always_inline)) { weigh(b * kRowsT + 32, masked, z, dz, j); });
      arrive(b + 1, next);
      move(row_own, row_rot, buf, next);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) rows_next(next, 0, j, kAhead);
      const From f = source(min(b + 2, b_end - 1), buf == 0 ? kRing - 1 : buf - 1);
      int ln = lane;
      asm volatile("" : "+v"(ln));
      if (f.last < kRowsT - 1) hold(f.last);
      products(next, 0, z, dz, [&](int j) __attribute__((always_inline)) {
        if (j % 2 == 1 && j / 2 < kAllCopies) copy_piece(f, j / 2, ln);
        early((b + 1) * kRowsT, masked, z, j);
        cols_next(buf, 1, j, KS + KO);
      });
      if constexpr (kAllCopies > (KS + KO) / 2) copy_piece(f, kAllCopies - 1, ln);
      mask((b + 1) * kRowsT, z);
      additions(buf, 1, [&](int j) __attribute__((always_inline)) {
        weigh((b + 1) * kRowsT, masked, z, dz, j);
        rows_next(next, 1, j, kSlots);
      });
      move(col_own, col_rot, buf, next);
      ++b;
      buf = next;
    };
    if constexpr (!KEYS)
      while (b + 1 < b_end && !is_masked(b + 1)) step(std::false_type{});
    while (b + 1 < b_end) step(std::true_type{});
    first(std::true_type{});
    additions(buf, 0, [&](int j) __attribute__((always_inline)) {
      weigh(b * kRowsT + 32, std::true_type{}, z, dz, j);
      cols_next(buf, 1, j, kSlots);
    });
    additions(buf, 1, [](int) {});
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // the ring is used again below
  }

  // ------------------------------------------------ results
  // Lane (n, h) holds dims 32 i + 8 (e / 4) + 4 h + e % 4 of its row.  They leave by rows, through an area of the wave's
  // own in the ring: segments of 16 bytes, permuted by the row as above.  (Straight from the accumulators a store
  // touches 32 rows; 15000 clocks a CTA instead of 5000.)
  sync();
  char* area = reinterpret_cast<char*>(&ring[0]) + wave * (kRing * sizeof(Tile) / kWaves);
  auto lay = [&](const f32x16& v, float f, int row, int i, bool half, char* base) {
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      uint2 p;
      p.x = pack_bf16x2(v[4 * e4 + 0] * f, v[4 * e4 + 1] * f);
      p.y = pack_bf16x2(v[4 * e4 + 2] * f, v[4 * e4 + 3] * f);
      const int seg = 4 * i + e4;
      *reinterpret_cast<uint2*>(base + (half ? row * 2 * kRot + 16 * (seg ^ half_mix(row)) : row * 2 * kDim + 16 * (seg ^ wide_mix(row))) +
                                8 * h) = p;
    }
  };
  // rows 0 .. 32 NT - 1 of the wave from the area
  auto leave = [&](const Grad& to, bool half, const char* base) {
    const int per = half ? 8 : 4;                  // rows per store
#pragma unroll 4
    for (int c = 0; c < 32 * NT / per; ++c) {
      const int r = per * c + (half ? lane >> 3 : lane >> 4), seg = half ? lane & 7 : lane & 15;
      const u32x4 v = *reinterpret_cast<const u32x4*>(
          base + (half ? r * 2 * kRot + 16 * (seg ^ half_mix(r)) : r * 2 * kDim + 16 * (seg ^ wide_mix(r))));
      if (w0 + r < limit) *reinterpret_cast<u32x4_at8*>(to.p + (base_x + w0 + r) * to.row + hd * to.head + 8 * seg) = v;
    }
  };
  constexpr int kWide = 32 * NT * 2 * kDim;        // bytes of the wave's rows of 128 elements
  static_assert(kWide * (KEYS ? 2 : 1) + 32 * NT * (KEYS ? 4 : 2) * kRot <= kRing * sizeof(Tile) / kWaves, "");
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = 32 * nt + n;
#pragma unroll
    for (int i = 0; i < KO / 2; ++i) lay(acc[i][nt], a.scale, row, i, false, area);
    if constexpr (KEYS) {
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i) lay(acc[ND + i][nt], 1.f, row, i, false, area + kWide);
#pragma unroll
      for (int i = KO / 2; i < ND; ++i)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)             // fp32: rows of 256 bytes
          *reinterpret_cast<f32x4*>(area + 2 * kWide + row * 4 * kRot + 16 * ((8 * (i - KO / 2) + 2 * e4 + h) ^ wide_mix(row))) =
              f32x4{acc[i][nt][4 * e4], acc[i][nt][4 * e4 + 1], acc[i][nt][4 * e4 + 2], acc[i][nt][4 * e4 + 3]};
    } else {
#pragma unroll
      for (int i = KO / 2; i < ND; ++i) lay(acc[i][nt], a.scale, row, i - KO / 2, true, area + kWide);
    }
  }
  wave_lds_order();                                // a lane stores what other lanes laid down
  leave(KEYS ? a.d_k : a.d_q, false, area);
  if constexpr (KEYS) {
    leave(a.d_v, false, area + kWide);
#pragma unroll 4
    for (int c = 0; c < 32 * NT / 4; ++c) {
      const int r = 4 * c + (lane >> 4), seg = lane & 15;
      const f32x4 v = *reinterpret_cast<const f32x4*>(area + 2 * kWide + r * 4 * kRot + 16 * (seg ^ wide_mix(r)));
      if (w0 + r < limit)
        *reinterpret_cast<f32x4*>(a.d_r + (static_cast<int64_t>(hd) * sq.total_kv_rows + base_x + w0 + r) * kRot + 4 * seg) = v;
    }
  } else {
    leave(a.d_e, true, area + kWide);
  }
}

// The shared part's gradient: the heads' sums, added in their order, times the
// scale.  A wave takes key rows, one element per lane.  Rows that no sequence
// owns get zeros, in d_kv too.
constexpr int64_t kSumCtas = 1 << 20;
__global__ __launch_bounds__(256) void latent_sum_kernel(const float* __restrict__ d_r, msa_seqs sq, int H, float scale,
                                                         uint16_t* __restrict__ d_kv, uint16_t* __restrict__ out, int64_t out_row) {
  const int lane = lane_id();
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; row < sq.total_kv_rows;
       row += static_cast<int64_t>(gridDim.x) * 4) {
    bool owned = false;
    for (int c = 0; c < sq.num_seqs && !owned; c += kWave) {
      bool here = false;
      if (c + lane < sq.num_seqs) {
        const int64_t start = seq_geom(sq, c + lane).kv_start;
        here = row >= start && row < start + tile_geom(sq, c + lane).kv_len;
      }
      owned = __ballot(here) != 0;
    }
    float sum = 0.f;
    if (owned) {
      for (int h0 = 0; h0 < H; h0 += 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d_r[(static_cast<int64_t>(min(h0 + i, H - 1)) * sq.total_kv_rows + row) * kRot + lane];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += h0 + i < H ? v[i] : 0.f;
      }
    } else {
      u32x4* y = reinterpret_cast<u32x4*>(d_kv + row * H * kPair);
      for (int i = lane; i < H * kPair / 8; i += kWave) y[i] = u32x4{};
    }
    out[row * out_row + lane] = static_cast<uint16_t>(pack_bf16x2(sum * scale, 0.f));
  }
}

// ---------------------------------------------------------------- host side
int validate_backward(const msa_seqs* seqs, int H) {
  int st = msa_host::validate_seqs(seqs);
  if (st != MSA_OK) return st;
  if (H < 1) return MSA_ERR_INVALID;
  if (seqs->block_table) return MSA_ERR_UNSUPPORTED;   // contiguous key side only
  if (H > 256) return MSA_ERR_UNSUPPORTED;
  if (seqs->total_q_rows * H >= (int64_t(1) << 31) || seqs->total_kv_rows * H >= (int64_t(1) << 31)) return MSA_ERR_UNSUPPORTED;
  return MSA_OK;
}
size_t stat_bytes(const msa_seqs* s, int H) { return msa_host::align_up(sizeof(uint4) * H * s->total_q_rows, 256); }
size_t work_bytes(const msa_seqs* s, int H) { return stat_bytes(s, H) + sizeof(float) * kRot * H * s->total_kv_rows; }

bool aligned(const void* p, int by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) == 0; }

}  // namespace

extern "C" size_t msa_latent_attn_backward_workspace_size(const msa_seqs* seqs, int num_heads) {
  return validate_backward(seqs, num_heads) == MSA_OK ? work_bytes(seqs, num_heads) : 0;
}

extern "C" int msa_latent_attn_backward(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                                        int64_t q_rope_stride, int64_t q_rope_head_stride, const void* kv, const void* k_rope,
                                        int64_t k_rope_stride, const void* o, const float* lse, const void* d_o,
                                        const msa_seqs* seqs, int num_heads, float softmax_scale, void* d_q, int64_t d_q_stride,
                                        int64_t d_q_head_stride, void* d_q_rope, int64_t d_q_rope_stride,
                                        int64_t d_q_rope_head_stride, void* d_kv, void* d_k_rope, int64_t d_k_rope_stride,
                                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int st = validate_backward(seqs, num_heads);
  if (st != MSA_OK) return st;
  const int H = num_heads;
  const int64_t T = seqs->total_q_rows, N = seqs->total_kv_rows;
  if (N == 0 && T == 0) return MSA_OK;
  if (T > 0 && (!q || !q_rope || !o || !lse || !d_o || !d_q || !d_q_rope)) return MSA_ERR_INVALID;
  if (N > 0 && (!kv || !k_rope || !d_kv || !d_k_rope)) return MSA_ERR_INVALID;
  // rows and heads of the results do not overlap
  auto apart = [&](int64_t row, int64_t head, int dim) {
    if ((T > 1 && row < dim) || (H > 1 && head < dim)) return false;
    return T <= 1 || H == 1 || row >= (H - 1) * head + dim || head >= (T - 1) * row + dim;
  };
  for (int64_t x : {q_stride, q_head_stride, q_rope_stride, q_rope_head_stride, k_rope_stride, d_q_stride, d_q_head_stride,
                    d_q_rope_stride, d_q_rope_head_stride, d_k_rope_stride})
    if (x < 0) return MSA_ERR_INVALID;
  if (T > 0 && (!apart(d_q_stride, d_q_head_stride, kDim) || !apart(d_q_rope_stride, d_q_rope_head_stride, kRot)))
    return MSA_ERR_INVALID;
  if (N > 1 && d_k_rope_stride < kRot) return MSA_ERR_INVALID;
  for (const void* x : {q, q_rope, kv, k_rope, o, d_o, static_cast<const void*>(d_kv)})
    if (!aligned(x, 16)) return MSA_ERR_UNSUPPORTED;
  if (!aligned(d_q, 8) || !aligned(d_q_rope, 8) || !aligned(d_k_rope, 2)) return MSA_ERR_UNSUPPORTED;
  if ((q_stride | q_head_stride | q_rope_stride | q_rope_head_stride | k_rope_stride) % 8 != 0) return MSA_ERR_UNSUPPORTED;
  if ((d_q_stride | d_q_head_stride | d_q_rope_stride | d_q_rope_head_stride) % 4 != 0) return MSA_ERR_UNSUPPORTED;
  for (int64_t x : {q_stride, q_rope_stride, k_rope_stride})
    if (x > (int64_t(1) << 24)) return MSA_ERR_UNSUPPORTED;           // 64 rows' offsets are 32 bits
  if (!workspace || workspace_bytes < work_bytes(seqs, H)) return MSA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return MSA_ERR_UNSUPPORTED;
  const auto* kvp = static_cast<const uint16_t*>(kv);
  auto* dkv = static_cast<uint16_t*>(d_kv);
  const int64_t kv_row = static_cast<int64_t>(H) * kPair, o_row = static_cast<int64_t>(H) * kDim;
  Args a{};
  a.q = Side{static_cast<const uint16_t*>(q), q_stride, q_head_stride};
  a.e = Side{static_cast<const uint16_t*>(q_rope), q_rope_stride, q_rope_head_stride};
  a.k = Side{kvp, kv_row, kPair};
  a.v = Side{kvp + kDim, kv_row, kPair};
  a.r = Side{static_cast<const uint16_t*>(k_rope), k_rope_stride, 0};
  a.o = Side{static_cast<const uint16_t*>(o), o_row, kDim};
  a.d_o = Side{static_cast<const uint16_t*>(d_o), o_row, kDim};
  a.lse = lse;
  a.d_q = Grad{static_cast<uint16_t*>(d_q), d_q_stride, d_q_head_stride};
  a.d_e = Grad{static_cast<uint16_t*>(d_q_rope), d_q_rope_stride, d_q_rope_head_stride};
  a.d_k = Grad{dkv, kv_row, kPair};
  a.d_v = Grad{dkv + kDim, kv_row, kPair};
  a.stat = static_cast<uint4*>(workspace);
  a.d_r = reinterpret_cast<float*>(static_cast<char*>(workspace) + stat_bytes(seqs, H));
  a.H = H;
  a.scale = softmax_scale;
  a.scale_log2 = softmax_scale * kLog2E;
  if (std::fabs(a.scale_log2) < kLeast) a.scale_log2 = kLeast;
  int64_t tiles;
  flash::Grid gr = flash::plan_grid(seqs, kRowTile, seqs->max_q_rows, &tiles);
  const bool few = tiles * H < kFewTiles;
  if (few) gr = flash::plan_grid(seqs, kRowTile / 2, seqs->max_q_rows, &tiles);
  // none where no sequence has a key: the rows that there are get zeros all the same
  const int64_t key_tiles = N == 0                ? 0
                            : seqs->num_seqs == 1 ? (std::min<int64_t>(seqs->max_kv_len, N) + kKeyTile - 1) / kKeyTile
                                                  : N / kKeyTile + seqs->num_seqs;
  if (std::max(tiles, key_tiles) * H >= (int64_t(1) << 24)) return MSA_ERR_UNSUPPORTED;     // a grid's limit
  if (T > 0)
    msa_prof::launch(few ? "latent_backward_q_narrow_kernel" : "latent_backward_q_kernel",
                     few ? latent_backward_kernel<false, 1> : latent_backward_kernel<false, 2>,
                     dim3(static_cast<unsigned>(tiles * H)), dim3(kThreads), 0, stream, a, *seqs, gr);
  if (key_tiles > 0)
    msa_prof::launch("latent_backward_kv_kernel", latent_backward_kernel<true, 1>,
                     dim3(static_cast<unsigned>(key_tiles * H)), dim3(kThreads), 0, stream, a, *seqs, gr);
  if (N > 0)
    msa_prof::launch("latent_sum_kernel", latent_sum_kernel, dim3(static_cast<unsigned>(std::min((N + 3) / 4, kSumCtas))), dim3(256), 0,
                     stream, static_cast<const float*>(a.d_r), *seqs, H, softmax_scale, dkv, static_cast<uint16_t*>(d_k_rope),
                     d_k_rope_stride);
  return msa_host::launch_status();
}
