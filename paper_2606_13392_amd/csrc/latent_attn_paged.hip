// Latent attention, absorbed form, on gfx950: causal attention of new rows over
// a paged cache that holds one vector of R latent and 64 rotated elements per
// token, keys of every head and (its latent part) their values.
//
// For row i, head h and token j:  S = scale (q_ih . c_j + e_ih . r_j),
// P = softmax_j S,  O_ih = sum_j P c_j.  All heads of a row meet the same keys,
// so a tile is up to 64 (row, head) pairs: several rows of few heads, or up to
// 64 heads of one row.
//
// A CTA of four waves streams a tile's keys 64 at a time through two LDS
// buffers that hold whole cache rows; each row comes from memory once for its
// score and its value.  Wave (kh, rh) forms the 32 x 32 scores of key half kh
// and row half rh (S^T = K Q^T, MFMA 32x32x16, Q in registers); the row maxima
// cross the two key halves in LDS, the weights go to LDS in bf16, and every wave
// adds O^T += C^T P^T for its quarter of the latent dimensions and all 64 rows.
// Splitting the value product by dimensions, not rows, keeps O in 128 registers
// a lane (512 x 64 in fp32 over four waves) and reads each latent from LDS twice
// for the scores and once for the values.
//
// The steps (64 keys of a tile) of all sequences are numbered through and dealt
// out evenly over the chip; a CTA forms the numbering from the lengths on the
// device.  Where a tile is shared by several CTAs each leaves its part in fp32,
// and latent_merge_kernel joins them by the log-sum-exp rule in key order.
#include <initializer_list>
#include <type_traits>

#include "flash_tile.h"
#include "latent_steps.h"

namespace {

using namespace msa;
using flash::copy16;
using flash::kLn_2;
using flash::kLog2E;
using flash::lds_address;
using flash::lds_tr4;
using flash::xor32f;
using steps::kKeys;
using steps::Share;
using steps::TileGeom;
using steps::tile_geom;

constexpr int kRot = 64;                 // elements of the shared rotated part
constexpr int kRows = 64;                // (row, head) pairs per tile
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kCtas = 256;               // one per CU: two buffers of keys fill its LDS
constexpr int kMinSteps = 4;             // steps per CTA, where there are few
constexpr int kAheadK = 6, kAheadV = 3;  // LDS operands requested so many products ahead

// A cache row in LDS: 16-byte segments, the low three bits of their number
// permuted by the row, so that 16 rows' reads of a segment, and the transposing
// reads of 4 rows x 4 segments, fall on all banks.  (A row is an odd multiple of
// 128 bytes: odd rows start in the other half of the banks.)
__device__ __forceinline__ int row_mix(int r) { return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3); }
// The weights in LDS: 64 keys = 8 segments per row.
__device__ __forceinline__ int p_seg(int r, int s) { return s ^ ((r >> 1) & 7); }

struct LatentPlan {
  int blocks;                            // head blocks of a row
  int heads;                             // heads per block, at most 64
  int rows;                              // query rows per tile (1 if there are several blocks)
  int ranges;                            // shares of the steps; each has `blocks` CTAs
  int min_steps;                         // per share
};
// What a share leaves of a tile that it does not have alone: slot 0 where it does
// not begin with the tile's first key, 1 where it does.
struct LatentParts {
  float* o;                              // [CTA][2][64 rows x R, in the accumulators' order], normalised
  float* lse;                            // [CTA][2][64], base 2
  int4* tile;                            // [CTA]: the tile in slot 1: sequence, tile, parts (0: none)
};

// T: cache elements, uint16_t = bf16 bits, uint8_t = E4M3 codes (o_scale
// multiplies O); R: latent elements.
template <typename T, int R>
__global__ __launch_bounds__(kThreads, 1) void latent_paged_kernel(
    const uint16_t* __restrict__ q, int64_t q_stride, int64_t q_head, const uint16_t* __restrict__ e, int64_t e_stride,
    int64_t e_head, const T* __restrict__ cache, msa_seqs sq, LatentPlan pl, LatentParts parts, int H, float scale_log2,
    uint32_t q_flip, float o_scale, uint16_t* __restrict__ o, float* __restrict__ lse) {
  constexpr bool kCodes = sizeof(T) == 1;
  constexpr int W = R + kRot;              // elements of a cache row
  constexpr int kSegs = W / 8;             // 16-byte segments of a row in LDS
  constexpr int KS = W / 16;               // k-steps of the scores
  constexpr int TD = R / 128;              // 32-dimension tiles of a wave's quarter
  constexpr int kRowBytes = W * 2;         // in LDS
  constexpr int kBuf = kKeys * kRowBytes;
  constexpr int kGroup = 16;               // a wave copies 16 keys of a step: never across a page's end
  constexpr int kSrcSegs = W * sizeof(T) / 16;
  constexpr int NC = kGroup * kSrcSegs / kWave;      // 16-byte pieces per lane and step
  static_assert(kGroup * kSrcSegs % kWave == 0, "");
  __shared__ __align__(16) uint16_t keys[2][kKeys * W];
  __shared__ __align__(16) uint16_t weights[kRows * kKeys];
  __shared__ float tops[2][kRows];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int n = lane & 31, h = lane >> 5;
  const int kh = wave & 1, rh = wave >> 1;
  // CTAs id and id + 8 are on one XCD: the head blocks of a share, which read the same keys
  const int id = static_cast<int>(blockIdx.x);
  const int block = (id >> 3) % pl.blocks, range = (id >> 3) / pl.blocks * 8 + (id & 7);
  const int cta = range * pl.blocks + block;

  Share sh(sq, pl.rows, pl.ranges, pl.min_steps, range);
  if (threadIdx.x == 0) parts.tile[cta] = make_int4(0, 0, 0, 0);

  // ------------------------------------------------ lane geometry
  const int tile_heads = min(pl.heads, H - block * pl.heads);     // of this block
  // K operand: row n of the wave's half, segment 2 st + h
  uint32_t k_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = (32 * kh + n) * kRowBytes + 16 * (((2 * i + h) & 7) ^ row_mix(n));
  // C^T operand: in each 16-lane group lane j addresses row k0 + j / 4, dims
  // n0 + 4 (j % 4) .. + 3, and receives rows k0 .. k0 + 3 of dim n0 + j
  uint32_t v_at[2][2];
  {
    const int gq = lane >> 4, jj = lane & 15;
    const int rl = 4 * h + (jj >> 2);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int seg = 4 * i + 2 * (gq & 1) + ((jj & 3) >> 1);
        v_at[i][b] = (rl + 8 * b) * kRowBytes + wave * (R / 4) * 2 + 16 * (seg ^ row_mix(rl + 8 * b)) + 8 * (jj & 1);
      }
  }
  const uint32_t lds_keys = lds_address(keys[0]);
  uint64_t piece_mixes = 0;                // row_mix of the row of each of the lane's pieces
#pragma unroll
  for (int c = 0; c < NC; ++c)
    piece_mixes |= static_cast<uint64_t>(row_mix((c * kWave + lane) / kSrcSegs)) << (3 * c);
  const int lg_page = 31 - __clz(sq.page_size);
  const int max_page = static_cast<int>(sq.total_kv_rows >> lg_page) - 1;

  for (; sh.more(); sh.next()) {
    const TileGeom& g = sh.g;
    const int64_t c_begin = sh.begin(), c_end = sh.end();
    const int t0 = sh.x * pl.rows, t_end = min(t0 + pl.rows, g.q_rows);
    const int base_p = g.kv_len - g.q_rows;                       // position of the sequence's first row
    const int seen = min(max(base_p + t_end, 0), g.kv_len);       // keys that the tile's last row sees
    const int visits = (seen + kKeys - 1) / kKeys;
    const int b_begin = static_cast<int>(min<int64_t>(c_begin, visits)), b_end = static_cast<int>(min<int64_t>(c_end, visits));
    const int nfree = max(0, base_p + t0 + 1) / kKeys;            // steps below see every row's keys
    const int pairs = (t_end - t0) * tile_heads;                  // rows of the tile
    const int32_t* table = sq.block_table + static_cast<int64_t>(sh.s) * sq.block_table_stride;

    // this lane's row of the scores, and of the two row halves of O
    const int mine = 32 * rh + n;
    const int my_t = t0 + min(mine, pairs - 1) / tile_heads;
    const int p = mine < pairs ? base_p + my_t : -1;

    // places of the wave's 16-key groups of 64 steps, one per lane, and of the next 64
    int w0 = b_begin, cur = 0, nxt = 0;
    const int last_group = g.kv_len > 0 ? (g.kv_len - 1) & ~15 : 0;
    auto fetch = [&](int step) {
      const int key = static_cast<int>(min<int64_t>(static_cast<int64_t>(step) * kKeys + 16 * wave, last_group));
      const int page = min(max(table[key >> lg_page], 0), max_page);
      return (page << lg_page) + (key & (sq.page_size - 1));
    };
    auto place = [&](int step) {             // steps in ascending order
      if (step - w0 >= kWave) {
        w0 += kWave;
        cur = nxt;
        nxt = fetch(w0 + kWave + lane);
      }
      return __builtin_amdgcn_readlane(cur, step - w0);
    };
    if (b_begin < b_end) {
      cur = fetch(w0 + lane);
      nxt = fetch(w0 + kWave + lane);
    }
    u32x4 raw[kCodes ? NC : 1];
    // Keys of step i: bf16 into buffer `buf` by copies of 1 KiB; codes into registers.
    // Piece c * 64 + lane of the wave's 16 rows is 16 bytes; by copy it lands at its own
    // number, so it is the segment that the row's permutation stores there.  (Rows are a
    // multiple of 8 segments, so the permutation is one of the piece's low three bits.)
    // Keys past the sequence's end repeat its last one: what memory holds there may be NaN.
    auto get = [&](int i, int buf) {
      const int64_t row = place(i);
      const char* src = reinterpret_cast<const char*>(cache) + row * (W * static_cast<int64_t>(sizeof(T)));
      const int key0 = i * kKeys + 16 * wave;
      const uint32_t dst = lds_keys + buf * kBuf + 16 * wave * kRowBytes;
      int piece = lane;
      asm volatile("" : "+v"(piece));        // offsets are formed here each time: held, they spill
      if (key0 + kGroup <= g.kv_len) {
        if constexpr (kCodes) {
#pragma unroll
          for (int c = 0; c < NC; ++c) raw[c] = *reinterpret_cast<const u32x4*>(src + 16 * piece + c * 1024);
        } else {
          uint64_t mixes = piece_mixes;
          asm volatile("" : "+v"(mixes));
#pragma unroll
          for (int c = 0; c < NC; ++c)
            copy16(src, 16 * ((c * kWave + piece) ^ (static_cast<uint32_t>(mixes >> (3 * c)) & 7)), dst + c * 1024);
        }
      } else {
        const int rem = g.kv_len - 1 - min(key0, last_group);     // last row of the group that may be read
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int r = (c * kWave + piece) / kSrcSegs, sg = (c * kWave + piece) % kSrcSegs;
          const uint32_t off = min(r, rem) * (W * sizeof(T));
          if constexpr (kCodes) raw[c] = *reinterpret_cast<const u32x4*>(src + off + 16 * sg);
          else copy16(src, off + 16 * (sg ^ row_mix(r)), dst + c * 1024);
        }
      }
    };
    auto put = [&](int buf) {                // codes, widened
      if constexpr (kCodes) {
        char* dst = reinterpret_cast<char*>(keys[buf]) + 16 * wave * kRowBytes;
        int piece = lane;
        asm volatile("" : "+v"(piece));
        uint64_t mixes = piece_mixes;
        asm volatile("" : "+v"(mixes));
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int d = 2 * (c * kWave + piece) + b;
            *reinterpret_cast<u32x4*>(dst + 16 * (d ^ (static_cast<int>(mixes >> (3 * c)) & 7))) =
                widen(u32x2{raw[c][2 * b], raw[c][2 * b + 1]});
          }
      }
    };

    // Q of the lane's row: k-step st holds elements 16 st + 8 h .. + 7
    bf16x8 bq[KS];
    {
      const int hd = block * pl.heads + min(mine, pairs - 1) % tile_heads;
      const int64_t row = g.q_begin + my_t;
      const uint16_t* qp = q + row * q_stride + hd * q_head + 8 * h;
      const uint16_t* ep = e + row * e_stride + hd * e_head + 8 * h;
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        u32x4 v = *reinterpret_cast<const u32x4*>(st < R / 16 ? qp + 16 * st : ep + 16 * (st - R / 16));
        if (mine >= pairs) v = u32x4{};
        bq[st] = __builtin_bit_cast(bf16x8, v ^ q_flip);
      }
    }
    f32x16 acc[TD][2];
#pragma unroll
    for (int i = 0; i < TD; ++i) acc[i][0] = acc[i][1] = f32x16{};
    float m_run[2] = {-INFINITY, -INFINITY}, l_run = 0.f;

    if (b_begin < b_end) {
      get(b_begin, 0);
      if constexpr (kCodes) {
        put(0);
        if (b_begin + 1 < b_end) get(b_begin + 1, 1);
      } else {
        if (b_begin + 1 < b_end) get(b_begin + 1, 1);
      }
    }
    for (int i = b_begin; i < b_end; ++i) {
      const int buf = (i - b_begin) & 1;
      const char* kb = reinterpret_cast<const char*>(keys[buf]);
      if constexpr (!kCodes) {               // the copies of step i have landed, those of i + 1 are under way
        if (i + 1 < b_end) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NC) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      f32x16 sc = {};
      {
        // fenced slots: LDS operands are requested kAheadK products before their use
        auto kread = [&](int st) {
          return ld_bf16x8(reinterpret_cast<const uint16_t*>(kb + k_at[st & 3] + (st >> 2) * 128));
        };
        bf16x8 kr[KS];
#pragma unroll
        for (int st = 0; st < kAheadK; ++st) kr[st] = kread(st);
#pragma unroll
        for (int st = 0; st < KS; ++st) {
          if (st + kAheadK < KS) kr[st + kAheadK] = kread(st + kAheadK);
          sc = mfma32x32x16(kr[st], bq[st], sc);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (i >= nfree) {
#pragma unroll
        for (int a = 0; a < 16; ++a) {
          const int key = i * kKeys + 32 * kh + 8 * (a >> 2) + 4 * h + (a & 3);
          sc[a] = key <= p ? sc[a] : -INFINITY;
        }
      }
      float top = sc[0];
#pragma unroll
      for (int a = 1; a < 16; ++a) top = fmaxf(top, sc[a]);
      top = fmaxf(top, xor32f(top));
      if (h == 0) tops[kh][mine] = top;
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      float alpha[2], neg[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float m_new = fmaxf(m_run[j], fmaxf(tops[0][32 * j + n], tops[1][32 * j + n]));
        const float mm = m_new == -INFINITY ? 0.f : m_new;        // rows with nothing visible yet
        alpha[j] = exp2_hw((m_run[j] - mm) * scale_log2);
        neg[j] = -mm * scale_log2;
        m_run[j] = m_new;
      }
      const float my_neg = rh ? neg[1] : neg[0];
      float sum = 0.f;
#pragma unroll
      for (int a = 0; a < 16; ++a) {
        sc[a] = exp2_hw(fmaf(sc[a], scale_log2, my_neg));
        sum += sc[a];
      }
      l_run = fmaf(l_run, rh ? alpha[1] : alpha[0], sum);
      // k-step u of the value product: keys 16 u + {4h + 0..3, 8 + 4h + 0..3}, as the scores hold them
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        uint4 w;
        w.x = pack_bf16x2(sc[8 * b + 0], sc[8 * b + 1]);
        w.y = pack_bf16x2(sc[8 * b + 2], sc[8 * b + 3]);
        w.z = pack_bf16x2(sc[8 * b + 4], sc[8 * b + 5]);
        w.w = pack_bf16x2(sc[8 * b + 6], sc[8 * b + 7]);
        *reinterpret_cast<uint4*>(weights + mine * kKeys + 8 * p_seg(mine, 2 * (2 * kh + b) + h)) = w;
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (__ballot(alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int td = 0; td < TD; ++td)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[td][j] *= alpha[j];
      }
      {
        constexpr int NU = kKeys / 16, NO = NU * TD;
        bf16x8 bp[NU][2], vr[NO];
        auto pread = [&](int us) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
            bp[us][j] = ld_bf16x8(weights + (32 * j + n) * kKeys + 8 * p_seg(n, 2 * us + h));
        };
        auto vread = [&](int k) {
          const int us = k / TD, td = k % TD;
          const char* a0 = kb + 16 * us * kRowBytes + (td >> 1) * 128;
          const uint2 x0 = lds_tr4(reinterpret_cast<const uint16_t*>(a0 + v_at[td & 1][0]));
          const uint2 x1 = lds_tr4(reinterpret_cast<const uint16_t*>(a0 + v_at[td & 1][1]));
          return __builtin_bit_cast(bf16x8, make_uint4(x0.x, x0.y, x1.x, x1.y));
        };
        pread(0);
#pragma unroll
        for (int k = 0; k < kAheadV; ++k) vr[k] = vread(k);
#pragma unroll
        for (int k = 0; k < NO; ++k) {
          const int us = k / TD, td = k % TD;
          if (td == 0 && us + 1 < NU) pread(us + 1);
          if (k + kAheadV < NO) vr[k + kAheadV] = vread(k + kAheadV);
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[td][j] = mfma32x32x16(vr[k], bp[us][j], acc[td][j]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if constexpr (kCodes) {
        if (i + 1 < b_end) {
          put(buf ^ 1);                      // its readers are behind the last barrier of step i - 1
          if (i + 2 < b_end) get(i + 2, buf);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      } else {
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the buffer's readers are done
        if (i + 2 < b_end) get(i + 2, buf);
      }
    }

    // ------------------------------------------------ the tile's rows, or the share's part of them
    l_run += xor32f(l_run);
    if (h == 0) tops[kh][mine] = l_run;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    float inv[2], lse2[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float l = tops[0][32 * j + n] + tops[1][32 * j + n];
      const bool empty = !(l > 0.f);
      inv[j] = empty ? 0.f : o_scale / l;
      lse2[j] = empty ? -INFINITY : m_run[j] * scale_log2 + __log2f(l);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // `tops` is free again
    const bool whole = b_begin == 0 && b_end == visits;
    if (whole && c_begin == 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = 32 * j + n;
        if (r >= pairs) continue;
        const int64_t head_row = (static_cast<int64_t>(g.q_begin) + t0 + r / tile_heads) * H + block * pl.heads + r % tile_heads;
        uint16_t* orow = o + head_row * R + wave * (R / 4) + 4 * h;
#pragma unroll
        for (int td = 0; td < TD; ++td)
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            uint2 w;
            w.x = pack_bf16x2(acc[td][j][4 * e4 + 0] * inv[j], acc[td][j][4 * e4 + 1] * inv[j]);
            w.y = pack_bf16x2(acc[td][j][4 * e4 + 2] * inv[j], acc[td][j][4 * e4 + 3] * inv[j]);
            *reinterpret_cast<uint2*>(orow + 32 * td + 8 * e4) = w;
          }
        if (wave == 0 && h == 0) lse[head_row] = lse2[j] * kLn_2;
      }
    } else if (b_begin < b_end) {
      const int slot = 2 * cta + (b_begin > 0 ? 0 : 1);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (32 * j + n >= pairs) continue;
        int at = wave * TD * 8 * kWave + lane;
        asm volatile("" : "+v"(at));         // as above
        f32x4* po = reinterpret_cast<f32x4*>(parts.o + static_cast<int64_t>(slot) * kRows * R) + at;
#pragma unroll
        for (int td = 0; td < TD; ++td)
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4)
            po[(td * 8 + 4 * j + e4) * kWave] =
                f32x4{acc[td][j][4 * e4], acc[td][j][4 * e4 + 1], acc[td][j][4 * e4 + 2], acc[td][j][4 * e4 + 3]} * inv[j];
        if (wave == 0 && h == 0) parts.lse[slot * kRows + 32 * j + n] = lse2[j];
      }
      if (b_begin == 0 && threadIdx.x == 0)
        parts.tile[cta] = make_int4(sh.s, sh.x, sh.parts(visits), 0);
    }
  }
}

// Joins the parts of a tile that several shares had: a = max LSE_c,
// LSE = a + log sum 2^(LSE_c - a), O = sum 2^(LSE_c - LSE) O_c, in key order.  Four
// dimensions of a row per thread, in the order of the parts.
template <int R>
__global__ __launch_bounds__(256) void latent_merge_kernel(msa_seqs sq, LatentPlan pl, LatentParts parts, int H,
                                                           uint16_t* __restrict__ o, float* __restrict__ lse) {
  constexpr int TD = R / 128;
  const int cta = static_cast<int>(blockIdx.x);
  const int4 what = parts.tile[cta];
  const int np = what.z;
  if (np < 1) return;
  const int block = cta % pl.blocks;
  const int unit = blockIdx.y * 256 + threadIdx.x;
  const int lane = unit & 63, rest = unit >> 6;
  const int e4 = rest & 3, j = (rest >> 2) & 1, td = (rest >> 3) % TD, wave = (rest >> 3) / TD;
  const int r = 32 * j + (lane & 31);
  const TileGeom g = tile_geom(sq, what.x);
  const int t0 = what.y * pl.rows, t_end = min(t0 + pl.rows, g.q_rows);
  const int tile_heads = min(pl.heads, H - block * pl.heads);
  if (r >= (t_end - t0) * tile_heads) return;
  auto slot = [&](int c) { return 2 * (cta + static_cast<int64_t>(c) * pl.blocks) + (c == 0 ? 1 : 0); };
  constexpr int kBatch = 8;
  float top = -INFINITY, sum = 0.f;
  f32x4 y{};
  for (int c0 = 0; c0 < np; c0 += kBatch) {
    float l[kBatch];
    f32x4 v[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int64_t at = slot(min(c0 + b, np - 1));
      l[b] = parts.lse[at * kRows + r];
      v[b] = reinterpret_cast<const f32x4*>(parts.o + at * kRows * R)[unit];
    }
    float m = top;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      l[b] = c0 + b < np ? l[b] : -INFINITY;
      m = fmaxf(m, l[b]);
    }
    const float base = m > -INFINITY ? m : 0.f;            // every part empty: all weights are zero
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
  const int64_t head_row = (static_cast<int64_t>(g.q_begin) + t0 + r / tile_heads) * H + block * pl.heads + r % tile_heads;
  uint2 w;
  w.x = pack_bf16x2(y[0] * inv, y[1] * inv);
  w.y = pack_bf16x2(y[2] * inv, y[3] * inv);
  *reinterpret_cast<uint2*>(o + head_row * R + wave * (R / 4) + 32 * td + 8 * e4 + 4 * (lane >> 5)) = w;
  if ((rest & ~4) == 0 && (lane >> 5) == 0) lse[head_row] = sum > 0.f ? (top + __log2f(sum)) * kLn_2 : -INFINITY;
}

// ---------------------------------------------------------------- host side
int validate_latent(const msa_seqs* seqs, int H, int R) {
  int st = msa_host::validate_seqs(seqs);
  if (st != MSA_OK) return st;
  if (H < 1 || R < 1) return MSA_ERR_INVALID;
  if (!seqs->block_table) return MSA_ERR_UNSUPPORTED;
  if (!msa_host::is_pow2(seqs->page_size) || seqs->page_size < 16 || seqs->page_size > 8192) return MSA_ERR_INVALID;
  if (R != 256 && R != 512) return MSA_ERR_UNSUPPORTED;
  if (H > 1024) return MSA_ERR_UNSUPPORTED;
  if (seqs->total_kv_rows >= (int64_t(1) << 31)) return MSA_ERR_UNSUPPORTED;
  return MSA_OK;
}

LatentPlan plan_of(int H) {
  LatentPlan pl{};
  pl.blocks = (H + kRows - 1) / kRows;
  pl.heads = (H + pl.blocks - 1) / pl.blocks;
  pl.rows = pl.blocks > 1 ? 1 : kRows / H;
  pl.ranges = std::max(8, kCtas / pl.blocks / 8 * 8);
  pl.min_steps = kMinSteps;
  return pl;
}
size_t slots_of(const LatentPlan& pl) { return static_cast<size_t>(2) * pl.ranges * pl.blocks; }
size_t part_bytes(const LatentPlan& pl, int R) {
  return slots_of(pl) * kRows * (R + 1) * sizeof(float) + slots_of(pl) / 2 * sizeof(int4);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int latent_paged(const void* q, int64_t q_stride, int64_t q_head, const void* e, int64_t e_stride, int64_t e_head,
                 const void* cache, bool fp8, float cache_scale, const msa_seqs* seqs, int H, int R, float softmax_scale,
                 void* o, float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int st = validate_latent(seqs, H, R);
  if (st != MSA_OK) return st;
  if (fp8 && !(cache_scale > 0.f && cache_scale < 3.0e38f)) return MSA_ERR_INVALID;
  if (seqs->total_q_rows == 0) return MSA_OK;
  if (!q || !e || !cache || !o || !lse) return MSA_ERR_INVALID;
  if (q_stride < 0 || q_head < 0 || e_stride < 0 || e_head < 0) return MSA_ERR_INVALID;
  for (const void* x : {q, e, cache, static_cast<const void*>(o)})
    if (!aligned16(x)) return MSA_ERR_UNSUPPORTED;
  if ((q_stride | q_head | e_stride | e_head) % 8 != 0) return MSA_ERR_UNSUPPORTED;
  const LatentPlan pl = plan_of(H);
  if (!workspace || workspace_bytes < part_bytes(pl, R)) return MSA_ERR_WORKSPACE;
  if (!aligned16(workspace)) return MSA_ERR_UNSUPPORTED;
  // in 64 bits: a scale of the codes far from 1 may cancel
  const flash::LogitScale scale = flash::logit_scale(static_cast<float>(static_cast<double>(softmax_scale) * cache_scale * kLog2E));
  LatentParts parts;
  parts.o = static_cast<float*>(workspace);
  parts.lse = parts.o + slots_of(pl) * kRows * R;
  parts.tile = reinterpret_cast<int4*>(parts.lse + slots_of(pl) * kRows);
  const unsigned ctas = static_cast<unsigned>(pl.ranges * pl.blocks);
  auto run = [&](auto elem, auto rank) {
    using T = decltype(elem);
    constexpr int RR = decltype(rank)::value;
    msa_prof::launch("latent_paged_kernel", latent_paged_kernel<T, RR>, dim3(ctas), dim3(kThreads), 0, stream,
                     static_cast<const uint16_t*>(q), q_stride, q_head, static_cast<const uint16_t*>(e), e_stride, e_head,
                     static_cast<const T*>(cache), *seqs, pl, parts, H, scale.log2, scale.q_flip, cache_scale,
                     static_cast<uint16_t*>(o), lse);
    msa_prof::launch("latent_merge_kernel", latent_merge_kernel<RR>, dim3(ctas, kRows * RR / 4 / 256), dim3(256), 0, stream,
                     *seqs, pl, parts, H, static_cast<uint16_t*>(o), lse);
  };
  using R256 = std::integral_constant<int, 256>;
  using R512 = std::integral_constant<int, 512>;
  if (fp8 && R == 512) run(uint8_t{}, R512{});
  else if (fp8) run(uint8_t{}, R256{});
  else if (R == 512) run(uint16_t{}, R512{});
  else run(uint16_t{}, R256{});
  return msa_host::launch_status();
}

}  // namespace

extern "C" size_t msa_latent_attn_paged_workspace_size(const msa_seqs* seqs, int num_heads, int latent_dim) {
  if (validate_latent(seqs, num_heads, latent_dim) != MSA_OK) return 0;
  return part_bytes(plan_of(num_heads), latent_dim);
}

extern "C" int msa_latent_attn_paged(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                                     int64_t q_rope_stride, int64_t q_rope_head_stride, const void* cache,
                                     const msa_seqs* seqs, int num_heads, int latent_dim, float softmax_scale, void* o,
                                     float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return latent_paged(q, q_stride, q_head_stride, q_rope, q_rope_stride, q_rope_head_stride, cache, false, 1.f, seqs,
                      num_heads, latent_dim, softmax_scale, o, lse, workspace, workspace_bytes, stream);
}

extern "C" int msa_latent_attn_paged_fp8(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                                         int64_t q_rope_stride, int64_t q_rope_head_stride, const void* cache,
                                         float cache_scale, const msa_seqs* seqs, int num_heads, int latent_dim,
                                         float softmax_scale, void* o, float* lse, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream) {
  return latent_paged(q, q_stride, q_head_stride, q_rope, q_rope_stride, q_rope_head_stride, cache, true, cache_scale, seqs,
                      num_heads, latent_dim, softmax_scale, o, lse, workspace, workspace_bytes, stream);
}
