// Dense causal GQA attention of new rows over a paged key / value cache on
// gfx950: a chunk of a prompt behind a cached context, a few draft rows, or
// one token per sequence; bf16 or E4M3.
//
// A CTA owns one KV group and a tile of consecutive query rows of one sequence
// (each of its 2, 4 or 8 waves holds 32 (query row, head) rows) and streams
// the sequence's keys, 64 at a time, through a double-buffered LDS ring one
// sub-block ahead: S^T = K Q^T and O^T += V^T P^T on MFMA 32x32x16, the online
// softmax of one sub-block between the O MFMAs of the one before (running
// maximum and sum per row in registers, fp32).  The layout of a sub-block in
// LDS and the transposing reads are those of flash_tile.h.
//
// Few tiles: the chip is then filled by a split of the keys.  The steps (64
// keys of one tile) of a group's tiles, one sequence after the other, are
// numbered through and dealt out evenly: CTA c of the group's gets steps
// c * per .. (c + 1) * per - 1, whatever lengths the sequences have, so a batch
// of ragged contexts ends everywhere at once.  Lengths are on the device, so
// every CTA forms the numbering itself (a wave's prefix sum over up to 256
// sequences).  Only a CTA's first and last tile can be shared with its
// neighbours; those leave their part in fp32, and merge_kernel joins them by
// the log-sum-exp rule.
//
// Pages: 16 .. 8192 rows, a power of two.  Each lane holds the place of one
// unit of min(page, 64) rows of the sequence, so 64 units' page ids arrive
// with one load, a window ahead of their use, and a sub-block's place comes
// from a lane read (pages of 64 rows and more) or a lane exchange (smaller
// ones).  Rows past the end of the sequence are never read: they repeat its
// last one, whose value is finite, at weight zero.
//
// E4M3 codes are widened to bf16, which is exact, on their way into LDS.  The
// 8-bit MFMA (32x32x64, twice the bf16 rate) on the codes themselves drops
// product bits some 2^-13 below the largest: LSE was off by up to 1.0e-4 on
// sequences of 5 - 34 keys (bf16: 1e-6).
//
// Tiles are bound by MFMA issue with the softmax between (64 heads on 8: 2 x 2048
// rows on 16K keys 1.78 - 1.92 ms by the card, 1.06 - 1.14 PFLOP/s), the few-row
// kernel by HBM reads (32 tokens on 4K - 60K keys 415 us, 5.7 TB/s; 64 on 32K
// 1.40 ms, 6.1 TB/s).
#include <initializer_list>

#include "flash_tile.h"

namespace {

using namespace msa;
using flash::kAhead;
using flash::kDim;
using flash::kLn_2;
using flash::kLog2E;
using flash::kSub;
using flash::k_seg;
using flash::lds_tr4;
using flash::Ring;
using flash::v_seg;
using flash::xor32f;

// global_load_lds: lane l's 16 bytes land at dst + 16 l (dst wave-uniform).  From
// inline assembly: the compiler cannot tell the ring's buffers apart and would
// wait for the copies just issued before the first read of the sub-block that
// has landed (2 x 2048 rows on 16K keys 2035 us instead of 1977); every step
// waits for them itself before its barrier.  M0 holds the LDS address, one wait
// state ahead of the copy.  It is a reserved register, which the compiler notes at
// every clobber: nothing else in these kernels uses it (LDS accesses do not need it,
// and no register is indexed by a variable).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<size_t>((__attribute__((address_space(3))) const void*)(p)));
}
__device__ __forceinline__ void copy16(const char* base, uint32_t offset, uint32_t lds) {   // base, lds wave-uniform
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(offset), "s"(base), "s"(lds) : "m0", "memory");
}
__device__ __forceinline__ void copy16(const char* src, uint32_t lds) {                      // src each lane its own
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(src), "s"(lds) : "m0", "memory");
}
#pragma clang diagnostic pop

// Places of a sequence's key rows in the pool, in units of min(page, 64) rows:
// a window of 64 units, one per lane, and the one behind it.  SMALL: pages of
// fewer than 64 rows.
template <bool SMALL>
struct PageWindow {
  const int32_t* table;                  // the sequence's block-table row
  int lg_unit, lg_page;
  int units;                             // units of the sequence
  int max_page;
  int w0;                                // first unit of `cur`
  int cur, nxt;                          // first row of the lane's unit

  __device__ __forceinline__ PageWindow(const msa_seqs& sq, int s, int kv_len) {
    table = sq.block_table + static_cast<int64_t>(s) * sq.block_table_stride;
    lg_page = 31 - __clz(sq.page_size);
    lg_unit = SMALL ? lg_page : 6;
    max_page = static_cast<int>(sq.total_kv_rows >> lg_page) - 1;
    units = ((kv_len - 1) >> lg_unit) + 1;
  }
  __device__ __forceinline__ int fetch(int unit) const {
    const int key = min(unit, units - 1) << lg_unit;
    const int page = min(max(table[key >> lg_page], 0), max_page);
    return (page << lg_page) + (key & ((1 << lg_page) - 1));
  }
  // sub-blocks from `sub` on; the sequence is not empty
  __device__ __forceinline__ void start(int sub) {
    w0 = sub << (6 - lg_unit);
    cur = fetch(w0 + lane_id());
    nxt = fetch(w0 + kWave + lane_id());
  }
  // Sub-block `sub`, at most 64 units past the last one asked for.  The place
  // of its row `row`: SMALL a row of the pool, each lane its own; else that of
  // the sub-block's first row, the same in every lane.
  __device__ __forceinline__ void advance(int sub) {
    if ((sub << (6 - lg_unit)) - w0 >= kWave) {
      w0 += kWave;
      cur = nxt;
      nxt = fetch(w0 + kWave + lane_id());
    }
  }
  __device__ __forceinline__ int place(int sub, int row) const {
    if constexpr (SMALL) {
      const int key = sub * kSub + row;
      return __shfl(cur, (key >> lg_unit) - w0) + (key & ((1 << lg_unit) - 1));
    } else {
      return __builtin_amdgcn_readlane(cur, sub - w0);
    }
  }
};

// How the steps are dealt out.
struct Plan {
  flash::Grid gr;                        // tiles of the unsplit grid
  int ctas;                              // CTAs per group that share its steps; 0: a CTA per tile and group
  int min_steps;                         // per CTA, where there are few
  int qt;                                // query rows per tile
};
constexpr int kMaxSplitSeqs = 256;       // four sequences per lane of the prefix sum

// A sequence with its lengths cut to the bounds that the host planned with.
__device__ __forceinline__ SeqGeom bounded_geom(const msa_seqs& sq, int s) {
  SeqGeom g = seq_geom(sq, s);
  g.kv_len = min(g.kv_len, sq.max_kv_len);
  g.q_rows = min(g.q_rows, sq.max_q_rows);
  return g;
}

// The numbering of a group's steps, formed by a wave: a tile of a sequence has
// as many as the sequence's last, at least one.
struct Steps {
  int cost[4];                           // steps of sequences 4 lane .. 4 lane + 3
  int q_begin[4], q_rows[4], kv_len[4];  // their geometry (paged: kv_start is unused)
  int before;                            // steps of all sequences before them
  int total, per;                        // of the group; of a CTA

  static __device__ __forceinline__ int blocks(const SeqGeom& g) { return max(1, (g.kv_len + kSub - 1) / kSub); }
  __device__ __forceinline__ Steps(const msa_seqs& sq, const Plan& pl) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * lane_id() + i;
      cost[i] = 0;
      q_begin[i] = INT32_MAX;
      q_rows[i] = kv_len[i] = 0;
      if (s < sq.num_seqs) {
        const SeqGeom g = bounded_geom(sq, s);
        q_begin[i] = g.q_begin;
        q_rows[i] = g.q_rows;
        kv_len[i] = g.kv_len;
        cost[i] = (max(g.q_rows, 0) + pl.qt - 1) / pl.qt * blocks(g);
      }
      sum += cost[i];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int x = __shfl_up(incl, d);
      if (lane_id() >= d) incl += x;
    }
    before = incl - sum;
    total = __builtin_amdgcn_readlane(incl, kWave - 1);
    per = max(pl.min_steps, (total + pl.ctas - 1) / pl.ctas);
  }
  // first step of each sequence, and behind the last one
  __device__ __forceinline__ void store(int (&first)[kMaxSplitSeqs + 1]) const {
    int x = before;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      first[4 * lane_id() + i] = x;
      x += cost[i];
    }
    if (lane_id() == kWave - 1) first[kMaxSplitSeqs] = x;
  }
  // sequence of step u < total (the same in every lane): the last that begins at or before it
  __device__ __forceinline__ int seq_of(int u) const {
    const int sum = cost[0] + cost[1] + cost[2] + cost[3];
    const int j = __ffsll(static_cast<unsigned long long>(__ballot(u >= before && u < before + sum))) - 1;
    int x = u - __builtin_amdgcn_readlane(before, j), i = 0;
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      const int c = __builtin_amdgcn_readlane(cost[e], j);
      if (i == e && x >= c) {
        x -= c;
        ++i;
      }
    }
    return 4 * j + i;
  }
  // sequence of a query row: the last that begins at or before it
  __device__ __forceinline__ int seq_of_row(int64_t row) const {
    int n = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) n += __popcll(__ballot(q_begin[e] <= row));
    return n;
  }
  __device__ __forceinline__ SeqGeom geom(int s) const {
    SeqGeom g{};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((s & 3) == e) {
        g.q_begin = __builtin_amdgcn_readlane(q_begin[e], s >> 2);
        g.q_rows = __builtin_amdgcn_readlane(q_rows[e], s >> 2);
        g.kv_len = __builtin_amdgcn_readlane(kv_len[e], s >> 2);
      }
    return g;
  }
  // first step of sequence s
  __device__ __forceinline__ int first(int s) const {
    int x = __builtin_amdgcn_readlane(before, s >> 2);
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < (s & 3)) x += __builtin_amdgcn_readlane(cost[e], s >> 2);
    return x;
  }
};

// The part of a tile that a CTA leaves to merge_kernel: 0 where it does not
// begin at the tile's first key, 1 where it does.  Each holds 32 * WAVES rows.
struct Parts {
  float* o;                              // [CTA][2][rows][128], normalised
  float* lse;                            // [CTA][2][rows], base 2
};

// Sub-block `sub` of a sequence's keys, as N of a thread's pieces see it.
template <bool SMALL, int N>
struct Rows {
  int at[SMALL ? N : 1];                 // SMALL: the pieces' rows in the pool; else the first row
  int last;                              // last row of the sub-block that the sequence has

  // row_of(c): the row of piece c
  template <typename F>
  __device__ __forceinline__ void find(PageWindow<SMALL>& pw, int sub, int kv_len, F row_of) {
    pw.advance(sub);
    last = kv_len - 1 - sub * kSub;
    if constexpr (SMALL) {
#pragma unroll
      for (int c = 0; c < N; ++c) at[c] = pw.place(sub, min(row_of(c), last));
    } else {
      at[0] = pw.place(sub, 0);
    }
  }
  // Piece c is 16 bytes at byte `seg` of row `row`: uniform base and lane offset
  // (whole sub-blocks: `off` = row * stride_b + seg, formed once).
  __device__ __forceinline__ const char* from(const char* base, uint32_t stride_b) const {
    return base + static_cast<int64_t>(at[0]) * stride_b;
  }
  __device__ __forceinline__ uint32_t offset(uint32_t off, uint32_t stride_b, int row, uint32_t seg) const {
    return last >= kSub - 1 ? off : static_cast<uint32_t>(min(row, last)) * stride_b + seg;
  }
  __device__ __forceinline__ const char* ptr(const char* base, uint32_t stride_b, int c, int row, uint32_t seg) const {
    if constexpr (SMALL) return base + static_cast<int64_t>(at[c]) * stride_b + seg;
    else return from(base, stride_b) + offset(row * stride_b + seg, stride_b, row, seg);
  }
};

// T: uint16_t = bf16 bits, uint8_t = E4M3 codes (o_scale multiplies O).
template <typename T, int WAVES, bool SMALL>
__global__ __launch_bounds__(WAVES* kWave, WAVES >= 4 ? 2 : 1) void paged_attn_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, msa_seqs sq, Plan pl, Parts parts, int H_q,
    int H_kv, float scale_log2, uint32_t q_flip, float o_scale, uint16_t* __restrict__ o, float* __restrict__ lse) {
  constexpr int kThreads = WAVES * kWave;
  constexpr bool kCodes = sizeof(T) == 1;
  constexpr int MT = kSub / 32;            // 32-key tiles of S^T
  constexpr int KS = kDim / 16;            // bf16: k-steps of S^T = K Q^T
  constexpr int kSegs = kDim * sizeof(T) / 16;        // 16-byte segments of a key row
  constexpr int N = kSub * kSegs / kThreads;          // pieces of 16 bytes per thread, sub-block and tensor
  constexpr int kPieceRows = kWave / kSegs;           // rows of a wave's piece
  __shared__ __align__(16) Ring ring;
  __shared__ int first[kMaxSplitSeqs + 1];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int n = lane & 31, h = lane >> 5;
  const int G = H_q / H_kv;
  const int qpw = 32 / G;                  // query rows per wave
  const int qt = WAVES * qpw;              // query rows per CTA
  const int jq = n / G, hh = n % G;
  const int r = static_cast<int>(blockIdx.x % H_kv);
  const int cta = static_cast<int>(blockIdx.x / H_kv);
  const char* kb = reinterpret_cast<const char*>(k + static_cast<int64_t>(r) * kDim);
  const char* vb = reinterpret_cast<const char*>(v + static_cast<int64_t>(r) * kDim);
  const uint32_t stride_b = static_cast<uint32_t>(H_kv * kDim * sizeof(T));

  // A thread's pieces: row piece_row(c) and a 16-byte segment.  By DMA lane l's
  // piece lands at 16 l of its wave's, so it takes the segment that the row's
  // permutation stores there (the permutations are involutions).
  auto piece_row = [&](int c) { return kPieceRows * (c * WAVES + wave) + lane / kSegs; };
  auto piece_seg = [&](int c, bool is_v) -> uint32_t {
    const int ra = piece_row(c), sg = lane % kSegs;
    return 16 * (kCodes ? sg : is_v ? v_seg(ra, sg) : k_seg(ra, sg));
  };
  uint32_t koff[N], voff[N];               // in whole sub-blocks of large pages
#pragma unroll
  for (int c = 0; c < N; ++c) {
    koff[c] = piece_row(c) * stride_b + piece_seg(c, false);
    voff[c] = piece_row(c) * stride_b + piece_seg(c, true);
  }
  const uint32_t lds_k = lds_address(ring.k[0]), lds_v = lds_address(ring.v[0]);
  // MFMA operand reads, relative to a ring buffer
  uint32_t ks_at[KS], vs_at[kDim / 32];
#pragma unroll
  for (int st = 0; st < KS; ++st) ks_at[st] = 2 * (n * kDim + 8 * k_seg(n, 2 * st + h));
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

  int u = 0, u_end = 1, s = 0;
  SeqGeom g{};
  if (pl.ctas > 0) {
    const Steps steps(sq, pl);
    u = cta * steps.per;
    u_end = min(steps.total, u + steps.per);
    if (u >= u_end) return;
    s = steps.seq_of(u);
    g = steps.geom(s);
    if (threadIdx.x < kWave) steps.store(first);
    __syncthreads();
  }
#pragma unroll 1
  while (u < u_end) {
    int tile, b_begin = 0, b_to = INT32_MAX;           // sub-blocks of this tile: to its last
    if (pl.ctas > 0) {
      if (s + 1 < sq.num_seqs && first[s + 1] <= u) {
        do ++s;
        while (s + 1 < sq.num_seqs && first[s + 1] <= u);
        g = bounded_geom(sq, s);
      }
      const int nb = Steps::blocks(g), off = u - first[s];
      tile = off / nb;
      b_begin = off - tile * nb;
      const int take = min(nb - b_begin, u_end - u);
      if (b_begin + take < nb) b_to = b_begin + take;
      u += take;
    } else {
      flash::locate_tile(sq, pl.gr, cta, qt, &s, &tile);
      g = bounded_geom(sq, s);
      u = u_end;
    }
    const int t0 = tile * qt;
    const int base_p = g.kv_len - g.q_rows;  // position of the sequence's first query row
    int t_end = min(t0 + qt, g.q_rows);
    t_end = static_cast<int>(min(static_cast<int64_t>(t_end), sq.total_q_rows - g.q_begin));
    if (t_end <= t0) continue;                              // uniform over the CTA
    const int p_last = base_p + t_end - 1;
    const int t = t0 + wave * qpw + jq;                     // this lane's query row in the sequence
    const bool valid = n < qpw * G && t < t_end;
    const int p = valid ? base_p + t : -1;
    const bool live = t0 + wave * qpw < t_end;              // the wave has rows
    // sub-blocks below nfree are visible to every row of the wave and need no mask
    const int nfree = (base_p + min(t0 + wave * qpw, t_end - 1) + 1) / kSub;
    const int64_t head_row = (static_cast<int64_t>(g.q_begin) + (valid ? t : t0)) * H_q + static_cast<int64_t>(r) * G + hh;
    const int b_all = p_last < 0 ? 0 : p_last / kSub + 1;
    const int b_end = min(b_to, b_all);
    if (b_begin > 0 && b_begin >= b_end) continue;          // the tile's rows see none of these keys

    f32x16 acc_o[kDim / 32];
#pragma unroll
    for (int i = 0; i < kDim / 32; ++i) acc_o[i] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;
    // P of the pending sub-block in bf16, as the B operand of O^T = V^T P^T:
    // k-step u covers keys 32(u/2) + 16(u%2) + {4h + e, 8 + 4h + e}, e = 0..3
    bf16x8 bp[kSub / 16];
    float alpha_pend = 0.f;                 // alpha of the sub-block whose P is in bp

    if (b_begin < b_end) {
      PageWindow<SMALL> pw(sq, s, g.kv_len);
      pw.start(b_begin);
      bf16x8 bq[KS];                          // the query rows, as the B operand of S^T
      // bf16 goes into LDS by DMA (copy); codes through registers (get, put)
      auto copy = [&](const char* base, const Rows<SMALL, N>& at, bool is_v, int buf) {
        const uint32_t lds = (is_v ? lds_v : lds_k) + buf * 2 * kSub * kDim + 1024 * wave;
#pragma unroll
        for (int c = 0; c < N; ++c) {
          if constexpr (SMALL)
            copy16(at.ptr(base, stride_b, c, 0, piece_seg(c, is_v)), lds + 1024 * WAVES * c);
          else
            copy16(at.from(base, stride_b), at.offset(is_v ? voff[c] : koff[c], stride_b, piece_row(c), piece_seg(c, is_v)),
                   lds + 1024 * WAVES * c);
        }
      };
      u32x4 rk[N], rv[N];
      auto get = [&](const char* base, const Rows<SMALL, N>& at, u32x4 (&raw)[N]) {
#pragma unroll
        for (int c = 0; c < N; ++c)
          raw[c] = *reinterpret_cast<const u32x4*>(at.ptr(base, stride_b, c, piece_row(c), 16 * (lane % kSegs)));
      };
      auto put = [&](const u32x4 (&raw)[N], bool is_v, uint16_t* dst) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const int ra = piece_row(c);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int sg = 2 * (lane % kSegs) + e;
            *reinterpret_cast<u32x4*>(dst + ra * kDim + 8 * (is_v ? v_seg(ra, sg) : k_seg(ra, sg))) =
                widen(u32x2{raw[c][2 * e], raw[c][2 * e + 1]});
          }
        }
      };
      Rows<SMALL, N> at_k, at_v;              // K is one sub-block ahead of V
      auto next_rows = [&](int sub) {
        at_v = at_k;
        if (sub < b_end) at_k.find(pw, sub, g.kv_len, piece_row);
      };

      // S^T = K Q^T on one sub-block: lane (n, h) gets keys 32i + 8(e/4) + 4h + e%4
      // of row n.  16 MFMA slots, each fenced off from the next so that the
      // compiler keeps the order; LDS operands are read kAhead slots ahead.
      auto scores = [&](const uint16_t* kbuf, f32x16 (&acc_s)[MT], auto beside) {
        const char* kbb = reinterpret_cast<const char*>(kbuf);
#pragma unroll
        for (int i = 0; i < MT; ++i) acc_s[i] = f32x16{};
        constexpr int NS = MT * KS;
        auto kread = [&](int j) -> bf16x8 {
          return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(kbb + ks_at[j % KS] + 2 * 32 * (j / KS) * kDim));
        };
        bf16x8 kr[NS];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) kr[j] = kread(j);
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          if (j + kAhead < NS) kr[j + kAhead] = kread(j + kAhead);
          acc_s[j / KS] = mfma32x32x16(kr[j], bq[j % KS], acc_s[j / KS]);
          beside(j);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      auto mask = [&](f32x16 (&acc_s)[MT], int key0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = key0 + 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
            acc_s[i][e] = key <= p ? acc_s[i][e] : -INFINITY;
          }
      };
      // eight weights as a B operand; their sum in fp32, as they are
      auto pack8 = [&](const f32x16& a, int e0, float& lsum) -> bf16x8 {
#pragma unroll
        for (int e = 0; e < 8; ++e) lsum += a[e0 + e];
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
      // V^T operand of k-step w, dim tile td, read down V's columns
      auto read_vt = [&](const uint16_t* vbuf, int w, int td) -> bf16x8 {
        const char* a0 = reinterpret_cast<const char*>(vbuf) + vs_at[td] + 2 * 16 * w * kDim;
        const uint2 x0 = lds_tr4(reinterpret_cast<const uint16_t*>(a0));
        const uint2 x1 = lds_tr4(reinterpret_cast<const uint16_t*>(a0 + 2 * 8 * kDim));  // rows +8: same permutation
        return __builtin_bit_cast(bf16x8, make_uint4(x0.x, x0.y, x1.x, x1.y));
      };
      // O^T += V^T P^T from one value sub-block in 16 fenced MFMA slots, beside(j)
      // after the j-th
      auto pv = [&](const uint16_t* vbuf, auto beside) {
        constexpr int NO = (kSub / 16) * (kDim / 32);
        auto vread = [&](int j) { return read_vt(vbuf, j / (kDim / 32), j % (kDim / 32)); };
        bf16x8 vr[NO];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) vr[j] = vread(j);
#pragma unroll
        for (int j = 0; j < NO; ++j) {
          if (j + kAhead < NO) vr[j + kAhead] = vread(j + kAhead);
          acc_o[j % (kDim / 32)] = mfma32x32x16(vr[j], bp[j / (kDim / 32)], acc_o[j % (kDim / 32)]);
          beside(j);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      // One sixteenth of a sub-block's softmax (raw scores; scale_log2 > 0 keeps
      // their order): j = 0, 1 the maximum, 2 .. 13 the weights, 14, 15 their sum
      // and the packing.
      struct Soft {
        float m0, m_new, alpha, neg, lsum;
        bf16x8 bp[kSub / 16];
      };
      auto soft_step = [&](Soft& z, f32x16 (&acc_s)[MT], int j) __attribute__((always_inline)) {
        if (j == 0) {
          z.m0 = -INFINITY;
          z.lsum = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) z.m0 = fmaxf(z.m0, acc_s[0][e]);
        } else if (j == 1) {
#pragma unroll
          for (int e = 0; e < 16; ++e) z.m0 = fmaxf(z.m0, acc_s[1][e]);
          z.m0 = fmaxf(z.m0, xor32f(z.m0));
          z.m_new = fmaxf(m_run, z.m0);
          const float mm = z.m_new == -INFINITY ? 0.f : z.m_new;   // rows with nothing visible yet
          z.alpha = exp2_hw((m_run - mm) * scale_log2);
          z.neg = -mm * scale_log2;
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
        for (int w = 0; w < kSub / 16; ++w) bp[w] = z.bp[w];
        alpha_pend = z.alpha;
      };

      // iteration b: K_{b+1} is in k[(b+1)&1], V_b in v[b&1]; after the S^T slots
      // each O^T slot carries one sixteenth of the next softmax, so the VALU works
      // while the MFMA pipe drains.
      auto step = [&](int b, auto masked_t) {
        constexpr bool masked = decltype(masked_t)::value;
        __builtin_amdgcn_s_waitcnt(0);        // this thread's copies of K_{b+1} and V_b have landed
        __syncthreads();                      // everyone's have, and block b-1's readers are done
        // the next copies go out between the last S^T slots: in front of them (some
        // sixty scalar and address instructions) they held up all eight waves (1977
        // us); after slots 6 and 10 1830, 12 and 14 1815 (E4M3: 325, 322)
        auto move_k = [&]() __attribute__((always_inline)) {
          if constexpr (kCodes) {
            if (b + 2 < b_end) put(rk, false, ring.k[b & 1]);
            next_rows(b + 3);
            if (b + 3 < b_end) get(kb, at_k, rk);
          } else {
            next_rows(b + 2);
            if (b + 2 < b_end) copy(kb, at_k, false, b & 1);
          }
        };
        auto move_v = [&]() __attribute__((always_inline)) {
          if constexpr (kCodes) {
            put(rv, true, ring.v[(b + 1) & 1]);
            if (b + 2 < b_end) get(vb, at_v, rv);
          } else {
            copy(vb, at_v, true, (b + 1) & 1);
          }
        };
        if (!live) {
          move_k();
          move_v();
          return;
        }
        rescale();
        __builtin_amdgcn_sched_barrier(0);
        f32x16 acc_s[MT];
        scores(ring.k[(b + 1) & 1], acc_s, [&](int j) __attribute__((always_inline)) {
          if (j == 12) move_k();
          if (j == 14) move_v();
        });
        Soft z;
        pv(ring.v[b & 1], [&](int j) __attribute__((always_inline)) {
          if (masked && j == 0) mask(acc_s, (b + 1) * kSub);
          soft_step(z, acc_s, j);
        });
        take(z);
      };

      // K and V of the first sub-block, K of the second; codes of the sub-blocks
      // after them wait in registers
      at_k.find(pw, b_begin, g.kv_len, piece_row);
      if constexpr (kCodes) {
        get(kb, at_k, rk);
        get(vb, at_k, rv);
        put(rk, false, ring.k[b_begin & 1]);
        put(rv, true, ring.v[b_begin & 1]);
        next_rows(b_begin + 1);
        if (b_begin + 1 < b_end) {
          get(kb, at_k, rk);
          get(vb, at_k, rv);
          put(rk, false, ring.k[(b_begin + 1) & 1]);
        }
        next_rows(b_begin + 2);
        if (b_begin + 2 < b_end) get(kb, at_k, rk);
      } else {
        copy(kb, at_k, false, b_begin & 1);
        copy(vb, at_k, true, b_begin & 1);
        next_rows(b_begin + 1);
        if (b_begin + 1 < b_end) copy(kb, at_k, false, (b_begin + 1) & 1);
      }
      {
        const T* qrow = q + head_row * kDim + 8 * h;
        Raw<T> rq[KS];
#pragma unroll
        for (int st = 0; st < KS; ++st) rq[st] = valid ? load_raw(qrow + 16 * st) : Raw<T>{};
#pragma unroll
        for (int st = 0; st < KS; ++st) bq[st] = __builtin_bit_cast(bf16x8, widen(rq[st]) ^ q_flip);
      }
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      if (live) {
        f32x16 acc_s[MT];
        scores(ring.k[b_begin & 1], acc_s, [](int) {});
        if (b_begin >= nfree) mask(acc_s, b_begin * kSub);
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
        pv(ring.v[b & 1], [](int) {});
      }
      __syncthreads();                        // the ring is free again
    }
    if (!valid) continue;
    const bool empty = !(l_run > 0.f);
    const float inv_l = empty ? 0.f : o_scale / l_run;
    const float lse2 = empty ? -INFINITY : m_run * scale_log2 + __log2f(l_run);
    // O^T tile td: lane (n, h) holds d = 32td + 8(e/4) + 4h + e%4 of row n
    if (b_begin > 0 || b_end < b_all) {
      const int64_t row = (2 * static_cast<int64_t>(blockIdx.x) + (b_begin > 0 ? 0 : 1)) * (32 * WAVES) + 32 * wave + n;
      float* dst = parts.o + row * kDim + 4 * h;
#pragma unroll
      for (int td = 0; td < kDim / 32; ++td)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
          *reinterpret_cast<f32x4*>(dst + 32 * td + 8 * e4) =
              f32x4{acc_o[td][4 * e4], acc_o[td][4 * e4 + 1], acc_o[td][4 * e4 + 2], acc_o[td][4 * e4 + 3]} * inv_l;
      if (h == 0) parts.lse[row] = lse2;
    } else {
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
    }
  }
}

// ---------------------------------------------------------------- few rows
// A tile of at most 32 (query row, head) rows: one token of a sequence, or a
// few draft rows.  Nothing but the keys' bytes costs then, and the time until
// the first of them are there: the CTA's four waves take sub-blocks of the same
// rows in turn, each through registers and LDS of its own (the next sub-block's
// keys are requested as soon as this one's have left the registers, its values
// likewise: up to 128 KiB under way per CU), and join their states in LDS.
constexpr int kRowWaves = 4;
constexpr int kRedStride = kDim + 4;     // fp32 row stride of the joined rows
struct WaveBuf {
  uint16_t k[kSub * kDim];
  uint16_t v[kSub * kDim];
};
static_assert(sizeof(WaveBuf) >= 32 * kRedStride * sizeof(float), "joined rows do not fit");

// Orders a wave's own LDS accesses (they complete in issue order; this keeps
// the compiler from moving them across).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <typename T, bool SMALL>
__global__ __launch_bounds__(kRowWaves* kWave, 1) void paged_rows_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, msa_seqs sq, Plan pl, Parts parts, int H_q,
    int H_kv, float scale_log2, uint32_t q_flip, float o_scale, uint16_t* __restrict__ o, float* __restrict__ lse) {
  constexpr int MT = kSub / 32, KS = kDim / 16;
  constexpr int kLanes = kDim * sizeof(T) / 16;        // lanes per key row
  constexpr int kRows = kWave / kLanes;                // key rows per load instruction
  constexpr int NL = kSub / kRows;                     // load instructions per sub-block and tensor
  __shared__ __align__(16) WaveBuf bufs[kRowWaves];
  __shared__ float state[kRowWaves][2][32];
  __shared__ int first[kMaxSplitSeqs + 1];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int n = lane & 31, h = lane >> 5;
  const int G = H_q / H_kv, qpw = 32 / G;
  const int jq = n / G, hh = n % G;
  const int r = static_cast<int>(blockIdx.x % H_kv);
  const int cta = static_cast<int>(blockIdx.x / H_kv);
  WaveBuf& buf = bufs[wave];
  const char* kb = reinterpret_cast<const char*>(k + static_cast<int64_t>(r) * kDim);
  const char* vb = reinterpret_cast<const char*>(v + static_cast<int64_t>(r) * kDim);
  const uint32_t stride_b = static_cast<uint32_t>(H_kv * kDim * sizeof(T));
  const int lrow = lane / kLanes, lseg = lane % kLanes;

  auto piece_row = [&](int c) { return c * kRows + lrow; };

  int u = 0, u_end = 1, s = 0;
  SeqGeom g{};
  if (pl.ctas > 0) {
    const Steps steps(sq, pl);
    u = cta * steps.per;
    u_end = min(steps.total, u + steps.per);
    if (u >= u_end) return;
    s = steps.seq_of(u);
    g = steps.geom(s);
    if (threadIdx.x < kWave) steps.store(first);
    __syncthreads();
  }
#pragma unroll 1
  while (u < u_end) {
    int tile, b_begin = 0, b_to = INT32_MAX;           // sub-blocks of this tile: to its last
    if (pl.ctas > 0) {
      if (s + 1 < sq.num_seqs && first[s + 1] <= u) {
        do ++s;
        while (s + 1 < sq.num_seqs && first[s + 1] <= u);
        g = bounded_geom(sq, s);
      }
      const int nb = Steps::blocks(g), off = u - first[s];
      tile = off / nb;
      b_begin = off - tile * nb;
      const int take = min(nb - b_begin, u_end - u);
      if (b_begin + take < nb) b_to = b_begin + take;
      u += take;
    } else {
      flash::locate_tile(sq, pl.gr, cta, qpw, &s, &tile);
      g = bounded_geom(sq, s);
      u = u_end;
    }
    const int t0 = tile * qpw;
    const int base_p = g.kv_len - g.q_rows;            // position of the sequence's first query row
    int t_end = min(t0 + qpw, g.q_rows);
    t_end = static_cast<int>(min(static_cast<int64_t>(t_end), sq.total_q_rows - g.q_begin));
    if (t_end <= t0) continue;
    const int p_last = base_p + t_end - 1;
    const int b_all = p_last < 0 ? 0 : p_last / kSub + 1;
    const int b_end = min(b_to, b_all);
    if (b_begin > 0 && b_begin >= b_end) continue;     // the tile's rows see none of these keys
    const bool valid = n < qpw * G && t0 + jq < t_end;
    const int p = valid ? base_p + t0 + jq : -1;
    const int nfree = (base_p + t0 + 1) / kSub;        // sub-blocks below it need no mask

    PageWindow<SMALL> pw(sq, s, g.kv_len);
    auto fetch = [&](const char* base, const Rows<SMALL, NL>& at, u32x4 (&dst)[NL]) {
#pragma unroll
      for (int c = 0; c < NL; ++c)
        dst[c] = *reinterpret_cast<const u32x4*>(at.ptr(base, stride_b, c, piece_row(c), 16 * lseg));
    };
    auto store = [&](const u32x4 (&src)[NL], bool is_v, uint16_t* dst) {
#pragma unroll
      for (int c = 0; c < NL; ++c) {
        const int ra = c * kRows + lrow;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<u32x4*>(dst + ra * kDim + 8 * (is_v ? v_seg(ra, lseg) : k_seg(ra, lseg))) = src[c];
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int seg = 2 * lseg + e;
            *reinterpret_cast<u32x4*>(dst + ra * kDim + 8 * (is_v ? v_seg(ra, seg) : k_seg(ra, seg))) =
                widen(u32x2{src[c][2 * e], src[c][2 * e + 1]});
          }
        }
      }
    };

    f32x16 acc_o[kDim / 32];
#pragma unroll
    for (int i = 0; i < kDim / 32; ++i) acc_o[i] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;
    u32x4 rk[NL], rv[NL];
    Rows<SMALL, NL> at;
    if (b_begin + wave < b_end) pw.start(b_begin + wave);
    // the query rows stay as they are loaded: turned into operands here, they
    // would be waited for before the first key is asked for
    Raw<T> rq[KS];
    {
      const T* qrow = q + ((static_cast<int64_t>(g.q_begin) + (valid ? t0 + jq : t0)) * H_q + static_cast<int64_t>(r) * G + hh) * kDim + 8 * h;
#pragma unroll
      for (int st = 0; st < KS; ++st) rq[st] = valid ? load_raw(qrow + 16 * st) : Raw<T>{};
    }
    // the first pass only requests: each load stands once in the code (16 KB
    // instead of 30, which every launch reads anew)
#pragma unroll 1
    for (int b = b_begin + wave - kRowWaves; b < b_end; b += kRowWaves) {
      const bool now = b >= b_begin, more = b + kRowWaves < b_end;
      wave_lds_order();
      if (now) store(rk, false, buf.k);
      if (more) {
        at.find(pw, b + kRowWaves, g.kv_len, piece_row);
        fetch(kb, at, rk);
      }
      if (!now) {
        if (more) fetch(vb, at, rv);
        continue;
      }
      wave_lds_order();
      // S^T = K Q^T: lane (n, h) gets keys 32i + 8(e/4) + 4h + e%4 of row n
      f32x16 acc_s[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        acc_s[i] = f32x16{};
#pragma unroll
        for (int st = 0; st < KS; ++st)
          acc_s[i] = mfma32x32x16(ld_bf16x8(buf.k + (32 * i + n) * kDim + 8 * k_seg(n, 2 * st + h)),
                                  __builtin_bit_cast(bf16x8, widen(rq[st]) ^ q_flip), acc_s[i]);
      }
      if (b >= nfree) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = b * kSub + 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
            acc_s[i][e] = key <= p ? acc_s[i][e] : -INFINITY;
          }
      }
      float bmax = -INFINITY;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) bmax = fmaxf(bmax, acc_s[i][e]);
      bmax = fmaxf(bmax, xor32f(bmax));
      const float m_new = fmaxf(m_run, bmax);
      const float mm = m_new == -INFINITY ? 0.f : m_new;   // rows with nothing visible yet
      const float alpha = exp2_hw((m_run - mm) * scale_log2), neg = -mm * scale_log2;
      float lsum = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          acc_s[i][e] = exp2_hw(fmaf(acc_s[i][e], scale_log2, neg));
          lsum += acc_s[i][e];
        }
      lsum += xor32f(lsum);
      l_run = l_run * alpha + lsum;
      m_run = m_new;
      if (__ballot(alpha != 1.f)) {
#pragma unroll
        for (int i = 0; i < kDim / 32; ++i) acc_o[i] *= alpha;
      }
      store(rv, true, buf.v);
      if (more) fetch(vb, at, rv);
      wave_lds_order();
      // O^T += V^T P^T; P^T as the B operand: k-step w covers keys 32(w/2) + 16(w%2) + {4h + e, 8 + 4h + e}
#pragma unroll
      for (int w = 0; w < kSub / 16; ++w) {
        const int i = w >> 1, e0 = 8 * (w & 1);
        uint4 pw4;
        pw4.x = pack_bf16x2(acc_s[i][e0 + 0], acc_s[i][e0 + 1]);
        pw4.y = pack_bf16x2(acc_s[i][e0 + 2], acc_s[i][e0 + 3]);
        pw4.z = pack_bf16x2(acc_s[i][e0 + 4], acc_s[i][e0 + 5]);
        pw4.w = pack_bf16x2(acc_s[i][e0 + 6], acc_s[i][e0 + 7]);
        const int row = 16 * w + 4 * h + ((lane & 15) >> 2);
#pragma unroll
        for (int td = 0; td < kDim / 32; ++td) {
          const int col = 32 * td + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          const uint16_t* a0 = buf.v + row * kDim + 8 * v_seg(row, col >> 3) + (col & 7);
          const uint2 x0 = lds_tr4(a0), x1 = lds_tr4(a0 + 8 * kDim);   // rows + 8: same permutation
          acc_o[td] = mfma32x32x16(__builtin_bit_cast(bf16x8, make_uint4(x0.x, x0.y, x1.x, x1.y)),
                                   __builtin_bit_cast(bf16x8, pw4), acc_o[td]);
        }
      }
    }
    // join: M = max m_w, L = sum l_w 2^(m_w - M), O = sum 2^(m_w - M) acc_w / L
    if (h == 0) {
      state[wave][0][n] = m_run;
      state[wave][1][n] = l_run;
    }
    __syncthreads();
    auto top = [&](int c) {
      float m = state[0][0][c];
#pragma unroll
      for (int w = 1; w < kRowWaves; ++w) m = fmaxf(m, state[w][0][c]);
      return m;
    };
    {
      const float f = m_run > -INFINITY ? exp2_hw((m_run - top(n)) * scale_log2) : 0.f;
      float* red = reinterpret_cast<float*>(&buf) + n * kRedStride + 4 * h;
#pragma unroll
      for (int td = 0; td < kDim / 32; ++td)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
          *reinterpret_cast<f32x4*>(red + 32 * td + 8 * e4) =
              f32x4{acc_o[td][4 * e4], acc_o[td][4 * e4 + 1], acc_o[td][4 * e4 + 2], acc_o[td][4 * e4 + 3]} * f;
    }
    __syncthreads();
    const int c = threadIdx.x >> 3, d0 = 16 * (threadIdx.x & 7);   // row c, dims d0 .. d0 + 15
    if (c < (t_end - t0) * G) {
      const float M = top(c);
      float L = 0.f;
      f32x4 x[4] = {};
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) {
        const float mw = state[w][0][c];
        L += mw > -INFINITY ? state[w][1][c] * exp2_hw((mw - M) * scale_log2) : 0.f;
        const float* red = reinterpret_cast<const float*>(&bufs[w]) + c * kRedStride + d0;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += *reinterpret_cast<const f32x4*>(red + 4 * i);
      }
      const bool empty = !(L > 0.f);
      const float inv_l = empty ? 0.f : o_scale / L;
      const float lse2 = empty ? -INFINITY : M * scale_log2 + __log2f(L);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] *= inv_l;
      if (b_begin > 0 || b_end < b_all) {
        const int64_t row = (2 * static_cast<int64_t>(blockIdx.x) + (b_begin > 0 ? 0 : 1)) * 32 + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(parts.o + row * kDim + d0 + 4 * i) = x[i];
        if (d0 == 0) parts.lse[row] = lse2;
      } else {
        const int64_t head_row = (static_cast<int64_t>(g.q_begin) + t0 + c / G) * H_q + static_cast<int64_t>(r) * G + c % G;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint4 w;
          w.x = pack_bf16x2(x[2 * i][0], x[2 * i][1]);
          w.y = pack_bf16x2(x[2 * i][2], x[2 * i][3]);
          w.z = pack_bf16x2(x[2 * i + 1][0], x[2 * i + 1][1]);
          w.w = pack_bf16x2(x[2 * i + 1][2], x[2 * i + 1][3]);
          *reinterpret_cast<uint4*>(o + head_row * kDim + d0 + 8 * i) = w;
        }
        if (d0 == 0) lse[head_row] = lse2 * kLn_2;
      }
    }
    __syncthreads();                      // the areas are free again
  }
}

// Joins the parts of the rows whose tile several CTAs had: a = max LSE_c,
// LSE = a + log sum 2^(LSE_c - a), O = sum 2^(LSE_c - LSE) O_c, in an order that
// the lengths fix.  A wave takes a (query row, group), its heads in turn: each
// of its four lane groups (16 lanes x 8 dims) has every fourth part of one head,
// or with HEADS = 4 all parts of a head of its own (tiles of many rows, which
// few CTAs share).
template <int HEADS>
__global__ __launch_bounds__(256) void merge_kernel(msa_seqs sq, Plan pl, Parts parts, int rows_per_tile, int H_q, int H_kv,
                                                    uint16_t* __restrict__ o, float* __restrict__ lse) {
  constexpr int kShare = 4 / HEADS;      // lane groups per head
  const int lane = lane_id();
  const int64_t pair = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave;
  const int64_t row = pair / H_kv;
  const int r = static_cast<int>(pair % H_kv);
  if (row >= sq.total_q_rows) return;
  const Steps steps(sq, pl);
  const int s = steps.seq_of_row(row);
  const SeqGeom g = steps.geom(s);
  const int t = static_cast<int>(row - g.q_begin);
  if (t >= g.q_rows) return;
  const int G = H_q / H_kv;
  const int tile = t / pl.qt, in_tile = t - tile * pl.qt;
  const int qpw = 32 / G;
  const int p_last = g.kv_len - g.q_rows + min((tile + 1) * pl.qt, g.q_rows) - 1;
  const int u0 = steps.first(s) + tile * Steps::blocks(g);
  const int visits = p_last < 0 ? 0 : p_last / kSub + 1;
  const int c0 = u0 / steps.per, c1 = visits < 1 ? c0 : min((u0 + visits - 1) / steps.per, pl.ctas - 1);
  if (c0 >= c1) return;                  // written by its one CTA
  const int np = c1 - c0 + 1, l16 = lane & 15, l4 = lane >> 4;
#pragma unroll 1
  for (int h0 = blockIdx.y * HEADS; h0 < G; h0 += gridDim.y * HEADS) {
    const int hh = min(h0 + (HEADS == 4 ? l4 : 0), G - 1);
    const int slot = 32 * (in_tile / qpw) + (in_tile % qpw) * G + hh;
    auto part_row = [&](int j) {         // of the CTA's two parts: the tile's beginning, or not
      return (2 * (static_cast<int64_t>(c0 + j) * H_kv + r) + (j == 0 ? 1 : 0)) * rows_per_tile + slot;
    };
    // parts in batches whose loads are under way together
    constexpr int kBatch = HEADS == 4 ? 4 : 8;
    float top = -INFINITY, sum = 0.f;
    f32x4 x0{}, x1{};
    for (int j0 = HEADS == 4 ? 0 : l4; j0 < np; j0 += kShare * kBatch) {
      float l[kBatch];
      f32x4 y[kBatch][2];
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        const int64_t at = part_row(min(j0 + kShare * e, np - 1));
        l[e] = parts.lse[at];
        const f32x4* src = reinterpret_cast<const f32x4*>(parts.o + at * kDim + 8 * l16);
        y[e][0] = src[0];
        y[e][1] = src[1];
      }
      float m = top;
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        l[e] = j0 + kShare * e < np ? l[e] : -INFINITY;
        m = fmaxf(m, l[e]);
      }
      const float base = m > -INFINITY ? m : 0.f;    // every part empty: all weights are zero
      const float f = exp2_hw(top - base);
      top = m;
      sum *= f;
      x0 *= f;
      x1 *= f;
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        const float w = exp2_hw(l[e] - base);
        sum += w;
        x0 += y[e][0] * w;
        x1 += y[e][1] * w;
      }
    }
    if constexpr (HEADS == 1) {
      float m = fmaxf(top, __uint_as_float(xor_lane_u32<16>(__float_as_uint(top))));
      m = fmaxf(m, __uint_as_float(xor_lane_u32<32>(__float_as_uint(m))));
      const float f = exp2_hw(top - (m > -INFINITY ? m : 0.f));
      top = m;
      auto join = [&](float v) {
        v *= f;
        v += __uint_as_float(xor_lane_u32<16>(__float_as_uint(v)));
        return v + __uint_as_float(xor_lane_u32<32>(__float_as_uint(v)));
      };
      sum = join(sum);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x0[i] = join(x0[i]);
        x1[i] = join(x1[i]);
      }
    }
    if (HEADS == 4 ? h0 + l4 >= G : l4 != 0) continue;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int64_t head_row = row * H_q + static_cast<int64_t>(r) * G + hh;
    uint4 w;
    w.x = pack_bf16x2(x0[0] * inv, x0[1] * inv);
    w.y = pack_bf16x2(x0[2] * inv, x0[3] * inv);
    w.z = pack_bf16x2(x1[0] * inv, x1[1] * inv);
    w.w = pack_bf16x2(x1[2] * inv, x1[3] * inv);
    *reinterpret_cast<uint4*>(o + head_row * kDim + 8 * l16) = w;
    if (l16 == 0) lse[head_row] = sum > 0.f ? (top + __log2f(sum)) * kLn_2 : -INFINITY;
  }
}

// ---------------------------------------------------------------- host side
int validate_paged(const msa_seqs* seqs, int H_q, int H_kv, int head_dim) {
  int st = msa_host::validate_seqs(seqs);
  if (st != MSA_OK) return st;
  if (H_q < 1 || H_kv < 1 || head_dim < 1 || H_q % H_kv != 0) return MSA_ERR_INVALID;
  if (!seqs->block_table) return MSA_ERR_UNSUPPORTED;   // a contiguous key side is msa_dense_attn's
  if (!msa_host::is_pow2(seqs->page_size) || seqs->page_size < 16 || seqs->page_size > 8192) return MSA_ERR_INVALID;
  if (head_dim != kDim) return MSA_ERR_UNSUPPORTED;
  if (H_q / H_kv > 16 || H_kv > 64) return MSA_ERR_UNSUPPORTED;
  if (seqs->total_q_rows * H_kv >= (int64_t(1) << 31)) return MSA_ERR_UNSUPPORTED;
  if (seqs->total_kv_rows >= (int64_t(1) << 31)) return MSA_ERR_UNSUPPORTED;
  return MSA_OK;
}

// Waves for the longest sequence's rows, and whether the keys are split.
//
// The chip holds one CTA of 8 waves, one of the few-row kernel, or two of 2 or 4
// waves per CU.  Unsplit, a call lasts as many steps as the longest sequence has
// sub-blocks, once per round of CTAs; split, its share of all steps and some ten
// more for the parts and their merge.  The lengths are on the device: several
// sequences are taken to have three quarters of the longest's on average.
// Measured, us split / whole (64 heads on 8): one token of one sequence on 512
// keys 13.6 / 11.2, 1024 13.7 / 17.0; 32 sequences 1024 31.8 / 26.8, 4096 102.8 /
// 97.4 (all of them equally long; of 4K - 60K 421 against what the longest takes,
// over 600); 512 rows on 1024 keys 37.1 / 35.1, 2048 52.7 / 59.7; 64 rows 512 22.1
// / 21.5, 1024 24.9 / 33.8.
// The steps counted are those of a tile that sees all of its sequence's keys, which
// holds for rows far behind a long context.  A prompt's early tiles see few: split,
// their CTAs end early and the others have full shares (3800 rows without context
// 382 us, 4200, which are too many tiles to be split, 319).  The same bound keeps
// decode batches of more than about 100 sequences on 8 groups whole, whatever their
// lengths (4K - 60K: 96 sequences 5.8 TB/s, 128 4.6).
constexpr int kFewRowsGain = 11, kTileGain = 9;      // steps that a split has to save
Plan plan_of(const msa_seqs* seqs, int H_q, int H_kv, int* waves, int64_t* ctas) {
  const int qpw = 32 / (H_q / H_kv);
  const int need = (seqs->max_q_rows + qpw - 1) / qpw;
  *waves = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 8;
  Plan pl{};
  pl.qt = *waves * qpw;
  int64_t tiles;
  pl.gr = flash::plan_grid(seqs, pl.qt, seqs->max_q_rows, &tiles);
  *ctas = tiles * H_kv;
  const int64_t held = *waves == 8 || *waves == 1 ? 256 : 512;
  const int64_t blocks = (static_cast<int64_t>(seqs->max_kv_len) + kSub - 1) / kSub;
  if (seqs->num_seqs > kMaxSplitSeqs || *ctas >= 4 * held || tiles * blocks >= (int64_t(1) << 30)) return pl;
  const int64_t per_seq = (seqs->max_q_rows + pl.qt - 1) / pl.qt;
  const int64_t work = std::min<int64_t>(tiles, seqs->num_seqs * per_seq) * H_kv;    // CTAs with rows, at most
  const int64_t rounds = (work + held - 1) / held;
  const int64_t mean4 = seqs->num_seqs > 1 ? 3 : 4;
  if (blocks * (4 * rounds * held - mean4 * work) <= 4 * held * (*waves == 1 ? kFewRowsGain : kTileGain)) return pl;
  pl.ctas = static_cast<int>(held / H_kv);
  pl.min_steps = 4;
  *ctas = static_cast<int64_t>(pl.ctas) * H_kv;
  return pl;
}
size_t part_bytes(int64_t ctas, int waves) { return sizeof(float) * 2 * ctas * 32 * waves * (kDim + 1); }

bool scale_ok(float x) { return x > 0.f && x < 3.0e38f; }   // finite and positive

int paged_attn(const void* q, const void* k, const void* v, bool fp8, float q_scale, float k_scale, float v_scale,
               const msa_seqs* seqs, int H_q, int H_kv, int head_dim, float softmax_scale, void* o, float* lse,
               void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int st = validate_paged(seqs, H_q, H_kv, head_dim);
  if (st != MSA_OK) return st;
  if (fp8 && (!scale_ok(q_scale) || !scale_ok(k_scale) || !scale_ok(v_scale))) return MSA_ERR_INVALID;
  if (seqs->total_q_rows == 0) return MSA_OK;
  if (!q || !k || !v || !o || !lse) return MSA_ERR_INVALID;
  for (const void* x : {q, k, v, static_cast<const void*>(o)})
    if (reinterpret_cast<uintptr_t>(x) & 15) return MSA_ERR_UNSUPPORTED;   // 16-byte pieces
  // in 64 bits: scales of the codes far from 1 may cancel
  const flash::LogitScale scale =
      flash::logit_scale(static_cast<float>(static_cast<double>(softmax_scale) * q_scale * k_scale * kLog2E));
  const int G = H_q / H_kv;
  int waves;
  int64_t ctas;
  const Plan pl = plan_of(seqs, H_q, H_kv, &waves, &ctas);
  if (ctas >= (int64_t(1) << 22)) return MSA_ERR_UNSUPPORTED;
  Parts parts{};
  if (pl.ctas > 0) {
    if (!workspace || workspace_bytes < part_bytes(ctas, waves)) return MSA_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return MSA_ERR_UNSUPPORTED;
    parts.o = static_cast<float*>(workspace);
    parts.lse = parts.o + 2 * ctas * 32 * waves * kDim;
  }
  auto launch = [&](const char* name, auto kernel, auto elem, int cta_waves) {
    using T = decltype(elem);
    msa_prof::launch(name, kernel, dim3(static_cast<unsigned>(ctas)), dim3(cta_waves * kWave), 0, stream,
                     static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v), *seqs, pl, parts, H_q, H_kv,
                     scale.log2, scale.q_flip, v_scale, static_cast<uint16_t*>(o), lse);
  };
  auto pick = [&](auto elem, auto small) {
    using T = decltype(elem);
    constexpr bool SMALL = decltype(small)::value;
    if (waves == 1) launch("paged_rows_kernel", paged_rows_kernel<T, SMALL>, elem, kRowWaves);
    else if (waves == 2) launch("paged_attn_kernel", paged_attn_kernel<T, 2, SMALL>, elem, 2);
    else if (waves == 4) launch("paged_attn_kernel", paged_attn_kernel<T, 4, SMALL>, elem, 4);
    else launch("paged_attn_kernel", paged_attn_kernel<T, 8, SMALL>, elem, 8);
  };
  const bool small = seqs->page_size < kSub;
  if (fp8 && small) pick(uint8_t{}, std::true_type{});
  else if (fp8) pick(uint8_t{}, std::false_type{});
  else if (small) pick(uint16_t{}, std::true_type{});
  else pick(uint16_t{}, std::false_type{});
  if (pl.ctas > 0) {
    // a wave per (row, group); where those are few one per head of them
    const int64_t pairs = seqs->total_q_rows * H_kv;
    const bool many = waves >= 4;
    const int by_head = pairs >= 4096 ? 1 : many ? (G + 3) / 4 : G;
    msa_prof::launch("paged_merge_kernel", many ? merge_kernel<4> : merge_kernel<1>,
                     dim3(static_cast<unsigned>((pairs + 3) / 4), by_head), dim3(256), 0, stream, *seqs, pl, parts, 32 * waves,
                     H_q, H_kv, static_cast<uint16_t*>(o), lse);
  }
  return msa_host::launch_status();
}

}  // namespace

extern "C" size_t msa_dense_attn_paged_workspace_size(const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                                                     int head_dim) {
  if (validate_paged(seqs, num_q_heads, num_kv_heads, head_dim) != MSA_OK) return 0;
  int waves;
  int64_t ctas;
  const Plan pl = plan_of(seqs, num_q_heads, num_kv_heads, &waves, &ctas);
  return pl.ctas > 0 ? part_bytes(ctas, waves) : 0;
}

extern "C" int msa_dense_attn_paged(const void* q, const void* k, const void* v, const msa_seqs* seqs, int num_q_heads,
                                    int num_kv_heads, int head_dim, float softmax_scale, void* o, float* lse,
                                    void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return paged_attn(q, k, v, false, 1.f, 1.f, 1.f, seqs, num_q_heads, num_kv_heads, head_dim, softmax_scale, o, lse,
                    workspace, workspace_bytes, stream);
}

extern "C" int msa_dense_attn_paged_fp8(const void* q, const void* k, const void* v, float q_scale, float k_scale,
                                        float v_scale, const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                                        int head_dim, float softmax_scale, void* o, float* lse, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream) {
  return paged_attn(q, k, v, true, q_scale, k_scale, v_scale, seqs, num_q_heads, num_kv_heads, head_dim, softmax_scale, o,
                    lse, workspace, workspace_bytes, stream);
}
