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
//
// Bound: 64 heads of one token do 121 operations for each byte of a bf16 cache, so
// memory and products both count.  32 tokens of 64 heads on 4K - 60K keys take 146 us
// (123 at the rate of a large copy): a step of 72 KiB takes 7100 clocks, 2200 of them
// waiting for memory, 5.1 TB/s while the steps run, the rest the start and the merge.
// Elsewhere a step's own work bounds, some 4600 clocks, of which the matrix units are
// busy 2180 (R = 256: 1150): a CTA has its CU alone, so nothing runs under the softmax, the
// barriers and the copies' issue.  At R = 512 that cannot be otherwise in this form: O and Q take
// 494 - 510 of 512 registers, two buffers of bf16 keys 153 of 160 KiB.  At R = 256 it can:
// 300 registers and 89 KiB (codes 69) leave room for a third buffer, or for more waves on other
// rows, which has not been tried.
// Draft rows of 128 heads on E4M3 keys, R = 512: 87 us (54 at the rate of a large
// product); four chunks of 20 - 150 rows of 32 heads, R = 256: 76, on E4M3 70 (30); the 32
// tokens on E4M3 114 - 118 (64), of R = 256 91 (68); one token
// on 8K keys 21, of which the steps are 6.  Eight waves, each with half of the scores'
// k-steps and an eighth of the dimensions, so that two share a SIMD, take 151, 104, 80 and
// 20 us for these four's kernels, four 147, 101, 78 and 20 (before the codes lay in LDS):
// the partial scores' way through LDS.
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
using flash::lds_tr8;
using flash::xor32f;
using steps::kKeys;
using steps::Share;
using steps::TileGeom;
using steps::tile_geom;

constexpr int kRot = 64;                 // elements of the shared rotated part
constexpr int kRows = 64;                // (row, head) pairs per tile
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kCtas = 256;               // one per CU: at R = 512 it fills the registers and the LDS
// The merge of 32 tokens on 4K - 60K keys takes 15.7 us with 256 CTAs, 11.3 with 1024, 11.0 with 4096; of four chunks
// of 32 heads, R = 256, 10.9, 7.6 and 8.2.
constexpr int kMergeCtas = 1024;
// Steps per CTA, where there are few.  One token of 64 heads on 8K keys, kernel and merge: 21.0 + 6.9 us with 1 (the
// merge has twice the parts), 18.4 + 5.3 with 2, 19.8 + 4.3 with 4.
constexpr int kMinSteps = 2;
constexpr float kSlack = 8.f;            // see the maxima below
constexpr int kAheadK = 6, kAheadV = 3;  // LDS operands requested so many products ahead

// A cache row in LDS: 16-byte segments, the low three bits of their number
// permuted by the row, so that 16 rows' reads of a segment, and the transposing
// reads of 4 rows x 4 segments, fall on all banks.  (A row is an odd multiple of
// 128 bytes: odd rows start in the other half of the banks.)
__device__ __forceinline__ int row_mix(int r) { return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3); }
// Codes: a row is an odd multiple of 64 bytes, so the low two bits, and half of the rows' reads lie in the other half.
template <typename T>
__device__ __forceinline__ int key_mix(int r) { return sizeof(T) == 1 ? (r >> 1) & 3 : row_mix(r); }
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
  int4* tile;                            // [CTA]: the tile in slot 1: first query row, (row, head) pairs, parts (0: none)
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
  constexpr int KS = W / 16;               // k-steps of the scores
  constexpr int TD = R / 128;              // 32-dimension tiles of a wave's quarter
  constexpr int kRowBytes = W * static_cast<int>(sizeof(T));       // in LDS as in memory
  constexpr int kBuf = kKeys * kRowBytes;
  constexpr int kGroup = 16;               // a wave copies 16 keys of a step: never across a page's end
  constexpr int kSrcSegs = kRowBytes / 16;
  constexpr int NC = kGroup * kSrcSegs / kWave;      // 16-byte pieces per lane and step
  constexpr int kEarly = (NC + 2) / 2;     // copies among the score products, the others among the value products
  static_assert(kGroup * kSrcSegs % kWave == 0, "");
  constexpr int kQBytes = kRows * W * 2;   // the tile's queries, once, behind the first buffer
  __shared__ __align__(16) char keys[kBuf + (kBuf > kQBytes ? kBuf : kQBytes)];
  __shared__ __align__(16) uint16_t weights[kRows * kKeys];
  __shared__ float tops[2][kRows];
  __shared__ __align__(16) int outgrown[kWaves];
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
  const uint32_t heads_inv = (65536 + tile_heads - 1) / tile_heads;
  auto per_row = [&](int r) { return static_cast<int>((static_cast<uint32_t>(r) * heads_inv) >> 16); };   // r / tile_heads, r < 64
  // K operand: row n of the wave's half; bf16: segment 2 st + h; codes: segment 2 j + h, whose 16 elements are those of
  // k-steps 2 j and 2 j + 1
  constexpr int kGroupSegs = kCodes ? 4 : 8;         // that the rows' permutation stays in
  uint32_t k_at[kGroupSegs / 2];
#pragma unroll
  for (int i = 0; i < kGroupSegs / 2; ++i) k_at[i] = (32 * kh + n) * kRowBytes + 16 * ((2 * i + h) ^ key_mix<T>(n));
  // C^T operand, a transposing read of 16 keys x 32 dims: in each 16-lane group lane j addresses (bf16) row k0 + j / 4, dims
  // n0 + 4 (j % 4) .. + 3, and receives rows k0 .. k0 + 3 of dim n0 + j, twice; (codes) row k0 + j / 2, dims n0 + 8 (j % 2)
  // .. + 7, and receives rows k0 .. k0 + 7
  uint32_t v_at[2][kCodes ? 1 : 2];
  {
    const int gq = lane >> 4, jj = lane & 15;
    const int rl = kCodes ? 8 * h + (jj >> 1) : 4 * h + (jj >> 2);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < (kCodes ? 1 : 2); ++b) {
        const int r = rl + 8 * b;
        if constexpr (kCodes)
          v_at[i][b] = r * kRowBytes + wave * (R / 4) + 16 * ((2 * i + (gq & 1)) ^ key_mix<T>(r)) + 8 * (jj & 1);
        else
          v_at[i][b] = r * kRowBytes + wave * (R / 4) * 2 + 16 * ((4 * i + 2 * (gq & 1) + ((jj & 3) >> 1)) ^ key_mix<T>(r)) + 8 * (jj & 1);
      }
  }
  const uint32_t lds_keys = lds_address(keys);
  uint64_t piece_mixes = 0;                // row_mix of the row of each of the lane's pieces
#pragma unroll
  for (int c = 0; c < NC; ++c)
    piece_mixes |= static_cast<uint64_t>(key_mix<T>((c * kWave + lane) / kSrcSegs)) << (3 * c);
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
    const int my_t = t0 + per_row(min(mine, pairs - 1));
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
    // Keys of a step go into a buffer by copies of 1 KiB.  Piece c * 64 + lane of the wave's 16 rows is 16 bytes; it
    // lands at its own number, so it is the segment that the row's permutation stores there.  (Rows are a
    // multiple of 8 segments, of 4 codes', so the permutation is one of the piece's low bits.)
    // Offsets are formed anew each time: held, they spill.
    auto source = [&](int i) { return reinterpret_cast<const char*>(cache) + place(i) * (W * static_cast<int64_t>(sizeof(T))); };
    // Pieces past the sequence's end repeat its last one (what memory holds there may be NaN), and behind the
    // last step all repeat one; no copy hangs on a branch.
    struct Source {
      const char* from;
      uint32_t limit;                        // offset of the last piece that may be read
    };
    auto keys_of = [&](int i) {
      const int ii = min(i, b_end - 1);
      const int rem = g.kv_len - 1 - min(ii * kKeys + 16 * wave, last_group);     // last row of the group that there is
      const uint32_t limit = min(rem + 1, kGroup) * static_cast<int>(W * sizeof(T)) - 16;
      return Source{source(ii), i < b_end ? limit : 0};
    };
    auto get = [&](const Source& src, int buf, int c, int piece, uint64_t mixes) __attribute__((always_inline)) {
      const uint32_t off = 16 * ((c * kWave + piece) ^ (static_cast<uint32_t>(mixes >> (3 * c)) & 7));
      copy16(src.from, min(off, src.limit), lds_keys + buf * kBuf + 16 * wave * kRowBytes + c * 1024);
    };
    auto get_all = [&](int i, int buf) {
      int piece = lane;
      uint64_t mixes = piece_mixes;
      asm volatile("" : "+v"(piece), "+v"(mixes));
      const Source src = keys_of(i);
#pragma unroll
      for (int c = 0; c < NC; ++c) get(src, buf, c, piece, mixes);
    };

    // Q of the tile's rows, through the second buffer: its own parts, 2 R bytes a row, segments in an order of the row
    // that keeps the reads below free of bank conflicts, then the rotated ones as in a key.  Rows behind the tile's
    // repeat its last.  (Straight from memory an operand's load touches 32 rows.)
    constexpr int kOwnSegs = R / 8;
    auto get_q = [&]() {
      auto row_of = [&](int r, int64_t* hd) {
        const int rr = min(r, pairs - 1), t = per_row(rr);
        *hd = block * pl.heads + rr - t * tile_heads;
        return static_cast<int64_t>(g.q_begin) + t0 + t;
      };
      int64_t hd;
      int ln = lane;
      asm volatile("" : "+v"(ln));
      if constexpr (kOwnSegs == kWave) {
        // a copy is one row: where it lies is worked out once for the wave (32 tokens on 4K - 60K keys 143 - 148 us instead of 148)
#pragma unroll 1
        for (int r = wave; r < kRows; r += kWaves) {
          const int64_t row = row_of(r, &hd);
          const uint64_t at = reinterpret_cast<uint64_t>(q + row * q_stride + hd * q_head);
          const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at));
          const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
          copy16(reinterpret_cast<const char*>(static_cast<uint64_t>(hi) << 32 | lo), 16 * (ln ^ (r & 15)), lds_keys + kBuf + 1024 * r);
        }
      } else {
#pragma unroll 1
        for (int c = wave; c < kRows * kOwnSegs / kWave; c += kWaves) {
          const int r = 2 * c + (ln >> 5), sg = ln % kOwnSegs;
          const int64_t row = row_of(r, &hd);
          copy16(reinterpret_cast<const char*>(q + row * q_stride + hd * q_head + 8 * (sg ^ (r & 15))), lds_keys + kBuf + 1024 * c);
        }
      }
#pragma unroll 1
      for (int c = wave; c < kRows * kRot / 8 / kWave; c += kWaves) {
        const int r = 8 * c + (ln >> 3), sg = ln & 7;
        const int64_t row = row_of(r, &hd);
        copy16(reinterpret_cast<const char*>(e + row * e_stride + hd * e_head + 8 * (sg ^ row_mix(r))),
               lds_keys + kBuf + kRows * R * 2 + 1024 * c);
      }
    };
    // k-step st holds elements 16 st + 8 h .. + 7 of the lane's row; codes: 32 (st / 2) + 16 h + 8 (st % 2) .. + 7
    bf16x8 bq[KS];
    auto read_q = [&]() {
      int r = mine;
      asm volatile("" : "+v"(r));
      const uint16_t* own = reinterpret_cast<const uint16_t*>(keys + kBuf) + r * R;
      const uint16_t* rot = reinterpret_cast<const uint16_t*>(keys + kBuf) + kRows * R + r * kRot;
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const int sg = kCodes ? 4 * (st >> 1) + 2 * h + (st & 1) : 2 * st + h;       // of 8 elements
        bq[st] = ld_bf16x8(st < R / 16 ? own + 8 * (sg ^ (r & 15)) : rot + 8 * ((sg - R / 8) ^ row_mix(r)));
      }
      if (q_flip != 0) {
#pragma unroll
        for (int st = 0; st < KS; ++st) bq[st] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, bq[st]) ^ q_flip);
      }
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        // (accumulation registers are for the sums; some of Q fits beside them)
        if (st < (TD == 4 ? 10 : 0)) asm volatile("" : "+a"(bq[st]));
        else asm volatile("" : "+v"(bq[st]));
      }
    };
    f32x16 acc[TD][2];
#pragma unroll
    for (int i = 0; i < TD; ++i) acc[i][0] = acc[i][1] = f32x16{};
    float m_run[2] = {-INFINITY, -INFINITY}, l_run = 0.f;

    if (b_begin < b_end) {
      get_q();
      get_all(b_begin, 0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      read_q();
    }
    // Step i: its keys are in buffer i - b_begin (mod 2).  The copies of step i + 1 go out
    // between the products of both kinds, one by one, so that requests are under
    // way all the time.
    for (int i = b_begin; i < b_end; ++i) {
      const int buf = (i - b_begin) & 1;
      const char* kb = keys + buf * kBuf;
      int piece = lane;
      uint64_t mixes = piece_mixes;
      asm volatile("" : "+v"(piece), "+v"(mixes));
      // everyone's keys of step i are in place, and the readers of step i - 1's are done
      asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      const Source next = keys_of(i + 1);
      f32x16 sc = {};
      {
        // fenced slots: LDS operands are requested kAheadK products before their use (codes: two products' with a read)
        constexpr int kPer = kCodes ? 2 : 1, kReads = KS / kPer, kFront = kAheadK / kPer;
        auto kread = [&](int j) {
          return *reinterpret_cast<const u32x4*>(kb + k_at[j & (kGroupSegs / 2 - 1)] + j / (kGroupSegs / 2) * 16 * kGroupSegs);
        };
        u32x4 kr[kReads];
#pragma unroll
        for (int j = 0; j < kFront; ++j) kr[j] = kread(j);
#pragma unroll
        for (int st = 0; st < KS; ++st) {
          const int j = st / kPer;
          if (st % kPer == 0 && j + kFront < kReads) kr[j + kFront] = kread(j + kFront);
          bf16x8 kk;
          if constexpr (kCodes) kk = widen_bf16x8(st & 1 ? u32x2{kr[j][2], kr[j][3]} : u32x2{kr[j][0], kr[j][1]});
          else kk = __builtin_bit_cast(bf16x8, kr[j]);
          sc = mfma32x32x16(kk, bq[st], sc);
          if (st % 3 == 1 && st / 3 < kEarly) get(next, buf ^ 1, st / 3, piece, mixes);
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
      // The maxima that the weights are relative to move only when one is outgrown by 2^kSlack: among 64 rows
      // some true maximum moves in most steps, and each time O would be rescaled (384 instructions a wave at
      // R = 512; 32 tokens on 4K - 60K keys 171 us instead of 149, chunks at R = 256 87 instead of 77).  Weights stay
      // below 2^kSlack, and their sums far from fp32's ends.  So a wave forms its weights before it knows the other
      // key half's maxima, and only where some wave has outgrown one are they formed again: a barrier and a way through
      // LDS less a step (32 tokens 153 us with them, 147 without).
      {
        const float m = rh ? m_run[1] : m_run[0];
        const bool grown = (top - m) * scale_log2 > kSlack;       // the first visible keys among them: m is -inf
        const uint64_t any = __ballot(grown);
        if (lane == 0) outgrown[wave] = any != 0;
      }
      float sum;
      auto weigh = [&]() __attribute__((always_inline)) {
        const float m = rh ? m_run[1] : m_run[0], neg = m == -INFINITY ? 0.f : -m * scale_log2;   // rows with nothing visible yet
        float w[16];
        sum = 0.f;
#pragma unroll
        for (int a = 0; a < 16; ++a) {
          w[a] = exp2_hw(fmaf(sc[a], scale_log2, neg));
          sum += w[a];
        }
        // k-step u of the value product, lanes h: keys 16 u + {4h + 0..3, 8 + 4h + 0..3}, as the scores hold them; codes:
        // 16 u + 8h + 0..7, as they are read
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          uint2 lo, hi;
          lo.x = pack_bf16x2(w[8 * b + 0], w[8 * b + 1]);
          lo.y = pack_bf16x2(w[8 * b + 2], w[8 * b + 3]);
          hi.x = pack_bf16x2(w[8 * b + 4], w[8 * b + 5]);
          hi.y = pack_bf16x2(w[8 * b + 6], w[8 * b + 7]);
          uint16_t* row = weights + mine * kKeys;
          const int u = 2 * kh + b;
          if constexpr (kCodes) {
            *reinterpret_cast<uint2*>(row + 8 * p_seg(mine, 2 * u) + 4 * h) = lo;
            *reinterpret_cast<uint2*>(row + 8 * p_seg(mine, 2 * u + 1) + 4 * h) = hi;
          } else {
            *reinterpret_cast<uint4*>(row + 8 * p_seg(mine, 2 * u + h)) = make_uint4(lo.x, lo.y, hi.x, hi.y);
          }
        }
      };
      weigh();
      constexpr int NU = kKeys / 16, NO = NU * TD;
      bf16x8 bp[NU][2];
      Raw<T> vr[NO];
      auto pread = [&](int us) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          bp[us][j] = ld_bf16x8(weights + (32 * j + n) * kKeys + 8 * p_seg(n, 2 * us + h));
      };
      auto vread = [&](int k) __attribute__((always_inline)) {
        const int us = k / TD, td = k % TD;
        const char* a0 = kb + 16 * us * kRowBytes + (td >> 1) * 16 * kGroupSegs;
        if constexpr (kCodes) {
          return lds_tr8(a0 + v_at[td & 1][0]);
        } else {
          const uint2 x0 = lds_tr4(reinterpret_cast<const uint16_t*>(a0 + v_at[td & 1][0]));
          const uint2 x1 = lds_tr4(reinterpret_cast<const uint16_t*>(a0 + v_at[td & 1][1]));
          return u32x4{x0.x, x0.y, x1.x, x1.y};
        }
      };
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      const int4 which = *reinterpret_cast<const int4*>(outgrown);
      pread(0);
#pragma unroll
      for (int k = 0; k < kAheadV; ++k) vr[k] = vread(k);
      // (the pins keep O in accumulation registers on the way around, else it is moved in every step)
      auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int td = 0; td < TD; ++td) asm volatile("" : "+a"(acc[td][0]), "+a"(acc[td][1]));
      };
      pin();
      if (__builtin_amdgcn_readfirstlane(which.x | which.y | which.z | which.w) != 0) {
        float alpha[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float m_new = fmaxf(tops[0][32 * j + n], tops[1][32 * j + n]);
          const bool grown = (m_new - m_run[j]) * scale_log2 > kSlack;
          alpha[j] = grown ? exp2_hw((m_run[j] - m_new) * scale_log2) : 1.f;
          m_run[j] = grown ? m_new : m_run[j];
        }
        l_run *= rh ? alpha[1] : alpha[0];
        weigh();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        pin();
        if (__ballot(alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
          for (int td = 0; td < TD; ++td)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[td][j] *= alpha[j];
          pin();
        }
        pread(0);
      }
      l_run += sum;
      {
#pragma unroll
        for (int k = 0; k < NO; ++k) {
          const int us = k / TD, td = k % TD;
          if (td == 0 && us + 1 < NU) pread(us + 1);
          if (k + kAheadV < NO) vr[k + kAheadV] = vread(k + kAheadV);
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[td][j] = mfma32x32x16(widen_bf16x8(vr[k]), bp[us][j], acc[td][j]);
          if (k % 2 == 0 && kEarly + k / 2 < NC) get(next, buf ^ 1, kEarly + k / 2, piece, mixes);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    // The buffers' readers are done, and every wave's copies, those behind the tile's last step among them, have landed:
    // the next tile's queries may go where another wave's were still under way, and no wave ends with one.
    asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

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
        const int64_t head_row = (static_cast<int64_t>(g.q_begin) + t0 + per_row(r)) * H + block * pl.heads + r - per_row(r) * tile_heads;
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
        parts.tile[cta] = make_int4(g.q_begin + t0, pairs, sh.parts(visits), 0);
    }
  }
}

// Joins the parts of a tile that several shares had: a = max LSE_c,
// LSE = a + log sum 2^(LSE_c - a), O = sum 2^(LSE_c - LSE) O_c.  A CTA forms the
// list of such tiles and takes every gridDim.x-th share of them.  Of many tiles a
// wave joins the parts of a piece, 4 dimensions of 32 rows in each half of it; of
// few the CTA's four waves have every fourth part, in order, and join in LDS.  One
// tile of 65 parts takes 5.3 us by the second way and 9.3 by the first, 8 sequences'
// draft rows of 128 heads (16 tiles and more) 13.8 and 9.0, 32 tokens 15.7 and 11.3.
constexpr int kManyTiles = 16;
template <int R>
__global__ __launch_bounds__(kThreads) void latent_merge_kernel(msa_seqs sq, LatentPlan pl, LatentParts parts, int H,
                                                                uint16_t* __restrict__ o, float* __restrict__ lse) {
  constexpr int TD = R / 128, kPieces = kRows * R / 4 / kWave;
  __shared__ int16_t list[kCtas];
  __shared__ int count[kWaves];
  __shared__ f32x4 side_o[kWaves][kWave];
  __shared__ float2 side_l[kWaves][kWave];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int ctas = pl.ranges * pl.blocks;  // at most kCtas = kThreads
  const bool has = static_cast<int>(threadIdx.x) < ctas && parts.tile[threadIdx.x].z > 0;
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
  // parts c0, c0 + step, ... of a piece, joined
  auto join = [&](int cta, int np, int piece, int r, int c0, int step, float& top, float& sum, f32x4& y) {
    constexpr int kBatch = 8;
    for (; c0 < np; c0 += step * kBatch) {
      float l[kBatch];
      f32x4 v[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int c = c0 + step * b;
        l[b] = -INFINITY;
        v[b] = f32x4{};
        if (c < np) {
          const int64_t at = 2 * (cta + static_cast<int64_t>(c) * pl.blocks) + (c == 0 ? 1 : 0);
          l[b] = parts.lse[at * kRows + r];
          v[b] = reinterpret_cast<const f32x4*>(parts.o + at * kRows * R)[piece * kWave + lane];
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
  };
  auto write = [&](const int4& what, int block, int piece, float top, float sum, const f32x4& y) {
    const int e4 = piece & 3, j = (piece >> 2) & 1, td = (piece >> 3) % TD, quarter = (piece >> 3) / TD;
    const int r = 32 * j + (lane & 31);
    const int tile_heads = min(pl.heads, H - block * pl.heads);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int64_t head_row = (static_cast<int64_t>(what.x) + r / tile_heads) * H + block * pl.heads + r % tile_heads;
    uint2 w;
    w.x = pack_bf16x2(y[0] * inv, y[1] * inv);
    w.y = pack_bf16x2(y[2] * inv, y[3] * inv);
    *reinterpret_cast<uint2*>(o + head_row * R + quarter * (R / 4) + 32 * td + 8 * e4 + 4 * (lane >> 5)) = w;
    if ((piece & ~4) == 0 && lane < 32) lse[head_row] = sum > 0.f ? (top + __log2f(sum)) * kLn_2 : -INFINITY;
  };
  const bool many = tiles >= kManyTiles;
  const int steps = many ? tiles * (kPieces / kWaves) : tiles * kPieces;
  for (int i = blockIdx.x; i < steps; i += gridDim.x) {
    const int n = many ? i * kWaves + wave : i;
    const int cta = list[n / kPieces], piece = n % kPieces;
    const int4 what = parts.tile[cta];
    const int r = 32 * ((piece >> 2) & 1) + (lane & 31);
    const bool mine = r < what.y;          // rows behind the tile's have no parts
    float top = -INFINITY, sum = 0.f;
    f32x4 y{};
    if (many) {                            // a wave has a piece
      if (!mine) continue;
      join(cta, what.z, piece, r, 0, 1, top, sum, y);
      write(what, cta % pl.blocks, piece, top, sum, y);
      continue;
    }
    if (mine) join(cta, what.z, piece, r, wave, kWaves, top, sum, y);
    side_o[wave][lane] = y;
    side_l[wave][lane] = make_float2(top, sum);
    __syncthreads();
    if (wave == 0 && mine) {
      float2 l[kWaves];
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        l[w] = side_l[w][lane];
        m = fmaxf(m, l[w].x);
      }
      const float base = m > -INFINITY ? m : 0.f;
      sum = 0.f;
      y = f32x4{};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_hw(l[w].x - base);
        sum = fmaf(l[w].y, f, sum);
        y += side_o[w][lane] * f;
      }
      write(what, cta % pl.blocks, piece, m, sum, y);
    }
    __syncthreads();                       // the side areas are free again
  }
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
    msa_prof::launch("latent_merge_kernel", latent_merge_kernel<RR>, dim3(kMergeCtas), dim3(kThreads), 0, stream,
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
