// Attention over the paged 8-bit cache: rows (t, g) of a sequence and cache head h, the query heads
// h*G + g at positions len - T + t, over the visible tokens i < len - T + t + 1 of its pages:
//   l_i = (q . c_i) s_page / sqrt(d),   out = sum_i softmax(l)_i v_i,   lse = ln sum_i exp(l_i).
//
// Bound by the read of the codes: 256 bytes a token and head against 2 R d products, so both products run
// on the tensor cores straight from the codes, which TMA brings into shared memory and nothing converts.
// Tiles are 128 tokens by R query rows, with the tokens on the 128 TMEM lanes:
//   S^T [tokens][rows] = K Q^T      A = K tile (K-major), B = the query rows
//   O^T [d][rows]      = V^T P^T    A = V tile as it lies (MN-major), B = the probabilities
// so a row block of 4 to 16 rows costs no padded lanes, a thread owns a token (and then a column d of the
// output), and 2 R and 3 R accumulator columns are read back. The 8-bit operands that are not codes are
// exact enough as sums of e4m3 pieces, each piece a column of its own:
//   q (8 significant bits) = hi + lo / 16, two pieces of 4 bits: exact but for elements below 2^-13 of
//     the row's largest, which keep an absolute error of 2^-21 of it;
//   p = hi + mid / 16 + lo / 256, three pieces of the probability against its own tile's maximum: a relative
//     2^-12 (2^-4 of the final bf16 rounding) down to 2^-14 of that maximum, an absolute 2^-26 of it below. Two
//     pieces would be the 2^-8 that bf16 probabilities have. Against the row's maximum every later tile of a
//     row with one dominating token would lie in the absolute part: the output of 700 equal tokens beside
//     one of probability 0.9993 and values 0 was off by 1.5e-2 (norm), and is by 5.6e-4 now. What a tile loses
//     is 2^-19 of its largest value at most (128 tokens of 2^-26), half the step of its page's codes.
//     Where a tile's pages have different value scales the pieces are of the probability times its page's, and
//     "maximum" means the largest of these products that the row sees: a page of far larger values costs the
//     others nothing where it is not seen (the newest drafts') or hardly counts.
// Statistics, sums and the output accumulate in fp32 registers: a tile's O^T is added to them, row by row,
// times exp(tile's maximum - maximum so far), so TMEM holds one tile's products and is never rescaled.
//
// Warps: the TMA producer (pages two tiles and scales one tile ahead), the MMA issuer (scores two tiles ahead of
// the value product), two that quantise the next block's query rows, and four softmax warps, eight for 16 rows
// (a thread is a token and 4 or 8 rows, then a column of the output). Two CTAs an SM, 96 KB of tiles each: with
// three V stages instead of four 16 rows take 57.0 us instead of 56.0 on 131072 tokens.
//
// Measured (device; rates as shares of a copy's 6780 GB/s): 64 sequences of 512 to 16384 tokens, 446 MB, 73 us = 90%;
// one of 131072, 269 MB, 46.4 us = 85%, 8 us of them the start (lengths, cut, first tiles) and the join of 38 parts a
// head; 24 of 500 to 8192 with 4 drafts each (16 rows), 125 MB, 33.1 us = 55%, bound by the chain of a tile (scores,
// maxima, meeting, exponentials, pieces, product: 2000 cycles a tile and SM, half of the issue slots empty); 16 of
// 96 to 700 8.6 us; one of 96 5.2 us, a chain of latencies. With more than 16 rows every block of 16 reads the pages
// again: 16 of 8192 with 8 drafts (32 rows), 271 MB, 93 us = 43%.
//
// The work is cut over the tokens: all (sequence, head, row block)s' tiles in one line, an equal share of it
// for each of two CTAs an SM, whatever the lengths (the lengths are read on the GPU: a captured call serves
// every later length). A block that falls to several CTAs is joined by the one that finishes last, from
// their fp32 parts in token order, so the sum does not depend on who that is.
#include "kve_internal.h"
#include "kve_line.cuh"
#include "kve_ptx.cuh"

namespace kve {
namespace {

constexpr uint32_t kKStages = 2, kVStages = 4;   // 96 KB of tiles a CTA; a K tile is done with two tiles before its V
constexpr int kTileBytes = kTileKeys * kHeadDim;
constexpr int kMostTilePages = kTileKeys / 16;

constexpr int kNoNan = 255;   // of positions 0 .. 126

// The value scale that leaves the sums is a tile's largest one, or a smaller one where its pages are further apart than
// this: a page's scale over it is then at least 2^-96 and, as long as they are not 2^192 apart, at most 2^96, so that
// a row's probabilities, which count from the largest product with a scale that it sees, stay within fp32.
constexpr float kMostLog = 96.f, kMostRatio = 7.92281625142643375935e28f;   // 2^96

constexpr int up16(int x) { return (x + 15) / 16 * 16; }

// R rows of a block; each of H groups of four softmax warps has R / H of them.
template <int R, int H>
struct ACfg {
  static constexpr int kRows = R / H;
  static constexpr int kThreads = 128 * (1 + H);    // producer, MMA issuer, query loader and one more; softmax
  static constexpr int kNs = up16(2 * R);           // columns of S^T: q's hi rows, then its lo rows
  static constexpr int kNp = up16(3 * R);           // columns of O^T: p's hi, mid and lo rows
  static constexpr int kOCol = 2 * kNs;             // two S^T, one O^T
  static constexpr int kTmemCols = 2 * kNs + kNp <= 64 ? 64 : 128;
  static constexpr uint32_t kIdescS = idesc_e4m3_f32(128, kNs, false);
  static constexpr uint32_t kIdescO = idesc_e4m3_f32(128, kNp, true);
  static constexpr size_t kV = size_t(kKStages) * kTileBytes;
  static constexpr size_t kQ = kV + size_t(kVStages) * kTileBytes;
  // blocks whose query rows are held, by part: four where they fit, so that batches of short sequences do not wait
  // for them (1000 of 64 tokens: 58.9 us against 62.9 with two)
  static constexpr uint32_t kQBufs = R > 8 ? 2 : 4;
  static constexpr size_t kQBytes = kNs * kHeadDim;
  static constexpr size_t kP = kQ + kQBufs * kQBytes;
  static constexpr size_t kCtl = kP + kNp * kTileKeys;
};

// How the line is cut (kve_line.cuh): a part costs about kPartTiles tiles besides its own (its query rows, the tensor
// cores' latency at its two ends, its output), and cuts that would leave fewer than `least` tiles of a block move to its
// end. That is 4 tiles where a share is 8 units at most and 2 where it is longer and evenness counts
// for more: 16 sequences of 96 to 700 tokens take 8.6 us with 4 against 9.4 with 2 and 10.8 with 1, 24 of 500
// to 8192 with 4 drafts each (a share of 16) 36.1 with 4 against 33.2 with 2 (32.6 with 1). With kPartTiles = 0 they
// take 10.6 and 35.5, and 64 sequences of 512 to 16384 76.4 instead of 72.0. No more CTAs take part than have
// kLeastUnits each, or a block.
constexpr int kPartTiles = 2;

template <int R, int H>
struct ACtl {
  uint64_t k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
  uint64_t m_full[kVStages];                   // the scales beside a V stage
  uint64_t s_full[2], q_full[ACfg<R, H>::kQBufs], q_empty[ACfg<R, H>::kQBufs];
  uint64_t p_full, o_full, meet[H], joined[H], drain;
  // of a tile's pages: the keys' scale, and the values' as 256 times a share of the one that leaves the sums, and that
  // share's log2
  float ks[kVStages][kMostTilePages], vs[kVStages][kMostTilePages], lvs[kVStages][kMostTilePages];
  float vtop[kVStages];                        // the one that leaves / 256
  uint32_t pages[kVStages];                    // bit j: page j of the tile holds tokens
  static constexpr uint32_t kQBufs = ACfg<R, H>::kQBufs;
  alignas(16) float red[2][4][R];              // row maxima of the warps, by tile parity
  // of a tile's rows: the maximum (logit and log2 of the value scale over the one that leaves), exp(old maximum - new),
  // exp(tile's maximum - new) in units of the row's sum, and by the tile's parity that times vtop
  // (each warp of the rows writes the same)
  alignas(16) float top[R], kept[R], share[R], back[2][R];
  float sum[kQBufs > 2 ? 2 : 1][4][R];         // row sums of the warps, at the end of a part (by its parity)
  // of the rows of a part in each query buffer: log2(e) / sqrt(d) / the power of two in the q pieces; tokens
  // that the row sees; where its output goes (elements of out, of lse), -1 for no row
  alignas(16) float qs[kQBufs][R];
  alignas(16) int seen[kQBufs][R];
  long long out_at[kQBufs][R];
  int lse_at[kQBufs][R];
  uint8_t nan_from[kQBufs][kHeadDim];          // see there
  Block split[2];                              // parts left for the join (each half writes the same)
  int last[2 * H], split_cta[2 * H];           // its parts, if they are all written; the CTA of the first
  Block blocks[kQBufs];                        // of the part in each query buffer; [0] first of the first part
  Cuts<kPartTiles> cuts;
  int ends[2];                                 // this CTA's tiles of the line
  int2 sums[ACfg<R, H>::kThreads / 32];        // tiles, sequences that have some
  uint32_t tmem_base;
  int abort, never;                            // never: stays 0 (waits that a given-up call still has to make)
};

template <int R, int H>
constexpr size_t attend_smem() {
  return ACfg<R, H>::kCtl + sizeof(ACtl<R, H>);
}

// The power of two that brings the largest magnitude (bf16 bits a, finite) into [128, 256), as fp32 bits.
__device__ __forceinline__ uint32_t piece_scale(uint32_t a) {
  const int e = 261 - static_cast<int>(a >> 7);   // 2^(7 - (x - 127)), biased
  return static_cast<uint32_t>(min(e, 253)) << 23;
}

// Three e4m3 pieces of two values of at most 256: x = hi + mid / 16 + lo / 256, each pair in 16 bits. The
// values are rounded to f16 first (2^-12 of them; below 2^-14 an absolute 2^-25), whose 11 bits three
// pieces of 4 hold, so that the rest is exact in packed f16, down to 2^-6: below that a piece is subnormal, and
// the sum of the three a multiple of 2^-17.
__device__ __forceinline__ void e4m3_pieces(float lo, float hi, uint32_t (&piece)[3]) {
  uint32_t x;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(hi), "f"(lo));
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
    piece[k] = c;
    if (k == 2) break;
    uint32_t v;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"(c));
    asm("{\n .reg .b32 d;\n sub.rn.f16x2 d, %1, %2;\n mul.rn.f16x2 %0, d, %3;\n}"
        : "=r"(x)
        : "r"(x), "r"(v), "r"(0x4c004c00u));   // 16
  }
}

__device__ __forceinline__ uint16_t to_bf16(float x) {
  uint16_t d;
  asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(d) : "f"(x));
  return d;
}

// ln of a row's sum given the log2 of its unit (no token seen: -inf; a NaN sum is not 0, its row is NaN).
__device__ __forceinline__ float log_sum(float top, float sum) {
  return sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + lg2(sum)) * 0.69314718056f;
}

static_assert(attend_smem<16, 2>() <= 113 * 1024 && attend_smem<8, 1>() <= 113 * 1024, "two CTAs an SM");

template <int R, int H>
__global__ void __launch_bounds__(ACfg<R, H>::kThreads, kAttendCtas)
cache_attend_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ AttendParams P) {
  using C = ACfg<R, H>;
  constexpr int N = C::kRows, kThreads = C::kThreads;
  extern __shared__ __align__(1024) uint8_t smem[];   // the tiles' swizzle counts from 1024 bytes
  ACtl<R, H>& ctl = *reinterpret_cast<ACtl<R, H>*>(smem + C::kCtl);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // row / group, for groups that are no power of two as for those that are
  const auto row_token = [&](int row) {
    return P.group_inverse ? static_cast<int>(__umulhi(static_cast<uint32_t>(row), P.group_inverse)) : row;
  };
  const int rows = P.q_tokens * P.c.group;
  const int blocks = (rows + R - 1) / R;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(&ctl.k_full[i], 1);
      mbar_init(&ctl.k_empty[i], 1);
    }
    for (int i = 0; i < kVStages; ++i) {
      mbar_init(&ctl.v_full[i], 1);
      mbar_init(&ctl.v_empty[i], 1);
      mbar_init(&ctl.m_full[i], 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&ctl.s_full[i], 1);
    for (int i = 0; i < C::kQBufs; ++i) {
      mbar_init(&ctl.q_full[i], 2);
      mbar_init(&ctl.q_empty[i], 4 * H + 1);   // the softmax warps, and the last scores
    }
    for (int i = 0; i < H; ++i) {
      mbar_init(&ctl.meet[i], 4);
      mbar_init(&ctl.joined[i], 1);
    }
    mbar_init(&ctl.p_full, 4 * H);
    mbar_init(&ctl.o_full, 1);
    mbar_init(&ctl.drain, 1);
    ctl.abort = ctl.never = 0;
    fence_mbar_init();
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  wait_previous_kernel();
  // The line's length, and the block in which this CTA's share starts: a run of sequences a thread (as line_share of kve_line.cuh)
  const int cap = P.c.max_pages << P.c.page_shift;
  const int per = (P.n_seq + kThreads - 1) / kThreads;
  const int s0 = min(static_cast<int>(threadIdx.x) * per, P.n_seq), s1 = min(s0 + per, P.n_seq);
  int mine = 0, filled = 0;   // tiles of one block each (2^30: too many), sequences that have some
  bool bad = false;
  for (int r = s0; r < s1; ++r) {
    const int len = __ldg(P.lens + r);
    bad |= len < 0 || len > cap;
    mine = min(mine + (min(max(len, 0), cap) + kTileKeys - 1) / kTileKeys, 1 << 30);
    filled += len > 0;
  }
  if (warp == 1) {
    __syncwarp();   // (the lanes leave the loop at different times)
    tmem_alloc(&ctl.tmem_base, C::kTmemCols);
    tmem_relinquish();
  }
  const int per_seq = P.c.heads * blocks;   // blocks of a sequence
  int front = mine, front_filled = filled;  // up to and with this thread's sequences
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, front, o), y = __shfl_up_sync(0xffffffffu, front_filled, o);
    if (lane >= o) {
      front = min(front + x, 1 << 30);
      front_filled += y;
    }
  }
  if (lane == 31) ctl.sums[warp] = make_int2(front, front_filled);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  int all_tiles = 0, all_filled = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const int2 x = ctl.sums[w];
    if (w < warp) {
      front = min(front + x.x, 1 << 30);
      front_filled += x.y;
    }
    all_tiles = min(all_tiles + x.x, 1 << 30);
    all_filled += x.y;
  }
  front -= mine;
  front_filled -= filled;
  // (tiles of 32 KB each: a line of 2^30 of them is no call that ends)
  const long long all_units = (static_cast<long long>(all_tiles) + all_filled * kPartTiles) * per_seq;
  const bool too_long = all_tiles >= 1 << 30 || all_units >= 1 << 30;
  if ((bad || too_long) && blockIdx.x == 0) atomicOr(P.err, kErrCheck);
  Cuts<kPartTiles> cuts;   // (in shared memory for the join: no registers' business in between)
  const int units = too_long ? 0 : static_cast<int>(all_units);
  cuts.set(units, max(min(max(units / kLeastUnits, all_filled * per_seq), static_cast<int>(gridDim.x)), 1));
  if (threadIdx.x == 0) ctl.cuts = cuts;
  if (cuts.units > 0 && static_cast<int>(blockIdx.x) < cuts.ctas) {
    // the thread that holds a cut's sequence says which tile of the line it is
    const int c0 = cuts.raw(blockIdx.x), c1 = cuts.raw(blockIdx.x + 1);
    int at = front * per_seq, index = front_filled * per_seq;   // tiles, blocks in front
    if (threadIdx.x == 0 && c1 == cuts.units) ctl.ends[1] = all_tiles * per_seq;
    for (int r = s0; r < s1; ++r) {
      const int len = seq_len(P, r), tiles = (len + kTileKeys - 1) / kTileKeys;
      if (tiles == 0) continue;
      const int unit = at + index * kPartTiles, size = tiles + kPartTiles;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = (e ? c1 : c0) - unit;
        if (c < 0 || c >= size * per_seq) continue;
        int b = c / size, j = c - b * size - kPartTiles;   // block of the sequence, tiles in front of the cut
        if (j < cuts.least) {
          j = 0;
        } else if (tiles - j < cuts.least) {
          j = 0;
          ++b;   // (a block's end is the next one's start)
        }
        ctl.ends[e] = at + b * tiles + j;
        if (e == 0) {
          Block f = {r, b / blocks, 0, len, tiles, at + b * tiles, index + b};
          f.rb = b - f.h * blocks;
          if (b == per_seq) {   // behind the sequence: the next one that is not empty, if there is one
            f.r = -1 - r;
          }
          ctl.blocks[0] = f;
        }
      }
      at += tiles * per_seq;
      index += per_seq;
    }
  } else if (threadIdx.x == 0) {
    ctl.ends[0] = ctl.ends[1] = 0;
  }
  __syncthreads();
  const int x0 = ctl.ends[0], x1 = ctl.ends[1];
  const bool works = x0 < x1;
  if (works && ctl.blocks[0].r < 0) {   // (for all threads)
    __syncthreads();
    if (threadIdx.x == 0) {
      Block f = ctl.blocks[0];
      f.r = -1 - f.r;
      f.h = f.rb = 0;
      do {
        f.len = seq_len(P, ++f.r);
        f.tiles = (f.len + kTileKeys - 1) / kTileKeys;
      } while (f.tiles == 0);
      ctl.blocks[0] = f;
    }
    __syncthreads();
  }
  const uint32_t tmem = ctl.tmem_base;
  const auto fail = [&]() {
    ctl.abort = 1;
    atomicOr(P.err, kErrWait);
  };

  if (warp == 0) {
    // ------------------------------------------------------------ producer: lane j the tile's page j
    if (works) {
      const int tile_pages = kTileKeys >> P.c.page_shift, page_bytes = P.c.page * kHeadDim;
      // pages run two tiles ahead and scales one: neither is waited for in the loop
      struct Ahead {
        Block b;
        int x, id;
        bool has;   // this lane's page holds tokens
      };
      const auto step = [&](Ahead a) {
        ++a.x;
        if (a.x < x1 && a.x == a.b.first + a.b.tiles) next_block(P, blocks, kTileKeys, a.b);
        const int j = (a.x - a.b.first) * tile_pages + lane;
        a.id = -1;
        a.has = a.x < x1 && lane < tile_pages && (j << P.c.page_shift) < a.b.len;
        if (a.has) a.id = __ldg(P.table + static_cast<int64_t>(a.b.r) * P.c.max_pages + j);
        return a;
      };
      const auto valid = [&](int id) { return id >= 0 && id < P.c.num_pages; };
      const auto scales = [&](const Ahead& a) {
        float2 f = make_float2(0.f, 0.f);
        if (valid(a.id)) {
          const int64_t block = static_cast<int64_t>(a.id) * P.c.heads + a.b.h;
          f.x = __ldg(P.c.k_scale + block);
          f.y = __ldg(P.c.v_scale + block);
        }
        return f;
      };
      Ahead now = step({ctl.blocks[0], x0 - 1, -1, false});
      Ahead then = step(now);
      float2 sc = scales(now);
      const uint32_t n = x1 - x0;
      uint32_t it = 0;
      // Pages of a call that reads more than L2 keeps anyway (8 tiles a share are 78 MB) leave it first: 64 ragged
      // sequences 74.9 -> 72.0 us, 131072 tokens 47.6 -> 46.0, and row blocks that read a page several times are no
      // slower (16 sequences of 8192 with 8 drafts 94.6 -> 93.0). Smaller caches may be there at the next call:
      // 16 of 96 to 700 tokens would be 0.1 slower.
      const uint64_t pol = n > 8 ? l2_policy_evict_first() : l2_policy_evict_normal();
      for (; it < n; ++it) {
        const uint32_t ks_at = it % kKStages, st = it % kVStages;
        const bool ok = valid(now.id);
        if (!ok && now.has) atomicOr(P.err, kErrCheck);
        const Ahead after = step(then);
        const float2 next_sc = scales(then);
        if (!warp_wait(&ctl.k_empty[ks_at], ((it / kKStages) & 1) ^ 1, P.wait_limit_ns, &ctl.abort) ||
            !warp_wait(&ctl.v_empty[st], ((it / kVStages) & 1) ^ 1, P.wait_limit_ns, &ctl.abort)) {
          if (lane == 0) fail();
          break;
        }
        const uint32_t mask = __ballot_sync(0xffffffffu, ok);
        if (lane == 0) {
          mbar_arrive_expect_tx(&ctl.k_full[ks_at], __popc(mask) * page_bytes);
          mbar_arrive_expect_tx(&ctl.v_full[st], __popc(mask) * page_bytes);
          ctl.pages[st] = mask;
        }
        __syncwarp();
        if (ok) {
          const int row = (now.id * P.c.heads + now.b.h) << P.c.page_shift;
          tma_load_2d_hint(smem + ks_at * kTileBytes + lane * page_bytes, &tm_k, 0, row, &ctl.k_full[ks_at], pol);
          tma_load_2d_hint(smem + C::kV + st * kTileBytes + lane * page_bytes, &tm_v, 0, row, &ctl.v_full[st], pol);
        }
        // one scale of the tile's values comes out of the sums; a token keeps the rest
        const float most = warp_max(sc.y), least = -warp_max(ok ? -sc.y : -INFINITY);
        const float top = fmaxf(fminf(most, least * kMostRatio), most * (1.f / kMostRatio));
        if (lane < kMostTilePages) {
          const float share = top > 0.f ? sc.y * rcp(top) : sc.y;
          ctl.ks[st][lane] = sc.x;
          ctl.vs[st][lane] = share * 256.f;
          ctl.lvs[st][lane] = fmaxf(lg2(share), -kMostLog);
        }
        if (lane == 0) ctl.vtop[st] = top * (1.f / 256.f);
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.m_full[st]);
        now = then;
        then = after;
        sc = next_sc;
      }
      // after a wait that ran out: the copies in flight end before the shared memory does
      if (ctl.abort && lane == 0) {
        for (uint32_t k = it > kKStages ? it - kKStages : 0; k < it; ++k)
          mbar_wait(&ctl.k_full[k % kKStages], (k / kKStages) & 1, P.wait_limit_ns, &ctl.never);
        for (uint32_t k = it > kVStages ? it - kVStages : 0; k < it; ++k)
          mbar_wait(&ctl.v_full[k % kVStages], (k / kVStages) & 1, P.wait_limit_ns, &ctl.never);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (works && lane == 0) {
      const uint32_t kaddr = smem_u32(smem), qaddr = kaddr + static_cast<uint32_t>(C::kQ);
      const uint32_t paddr = kaddr + static_cast<uint32_t>(C::kP);
      int end = x0;               // of the part's block
      const uint32_t n = x1 - x0;
      uint32_t part = 0xffffffffu;
      // S^T of tile `it`; it runs two tiles ahead of the probabilities
      const auto scores = [&](uint32_t it) -> bool {
        const int x = x0 + static_cast<int>(it);
        const uint32_t st = it % kKStages;
        if (x == end) {
          ++part;
          if (!mbar_wait(&ctl.q_full[part % C::kQBufs], (part / C::kQBufs) & 1, P.wait_limit_ns, &ctl.abort)) return false;
          end = ctl.blocks[part % C::kQBufs].first + ctl.blocks[part % C::kQBufs].tiles;
        }
        if (!mbar_wait(&ctl.k_full[st], (it / kKStages) & 1, P.wait_limit_ns, &ctl.abort)) return false;
        tc_fence_after();
        const uint64_t a = sw128_desc(kaddr + st * kTileBytes);
        const uint64_t b = sw128_desc(qaddr + part % C::kQBufs * static_cast<uint32_t>(C::kQBytes));
        const uint32_t d = tmem + (it & 1) * C::kNs;
#pragma unroll
        for (int j = 0; j < kHeadDim / 32; ++j)   // 32 elements of d a step: 32 bytes of a row
          tc_mma_e4m3(d, a + 2 * j, b + 2 * j, C::kIdescS, j > 0);
        tc_commit(&ctl.k_empty[st]);
        tc_commit(&ctl.s_full[it & 1]);
        if (x + 1 == x1 || x + 1 == end) tc_commit(&ctl.q_empty[part % C::kQBufs]);
        return true;
      };
      bool ok = scores(0) && (n == 1 || scores(1));
      for (uint32_t it = 0; ok && it < n; ++it) {
        const uint32_t st = it % kVStages;
        if (!mbar_wait(&ctl.v_full[st], (it / kVStages) & 1, P.wait_limit_ns, &ctl.abort) ||
            !mbar_wait(&ctl.p_full, it & 1, P.wait_limit_ns, &ctl.abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t vaddr = kaddr + static_cast<uint32_t>(C::kV) + st * kTileBytes;
#pragma unroll
        for (int j = 0; j < kTileKeys / 32; ++j)   // 32 tokens a step: four 8-row groups of V, of P
          tc_mma_e4m3(tmem + C::kOCol, sw128_mn_desc(vaddr + 4096u * j, kTileBytes, 1024),
                      plain_mn_desc(paddr + 512u * j, 128, 16 * kTileKeys), C::kIdescO, j > 0);
        tc_commit(&ctl.v_empty[st]);
        tc_commit(&ctl.o_full);
        if (it + 2 < n) ok = scores(it + 2);
      }
      if (!ok) {
        fail();
        tc_commit(&ctl.drain);   // what was issued ends before TMEM is given back
        mbar_wait(&ctl.drain, 0, P.wait_limit_ns, &ctl.never);
      }
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------ query rows, a block ahead
    // Two e4m3 pieces, K-major with the 128-byte swizzle: 16 lanes a row, 8 elements each; four rows at once.
    if (works) {
      uint8_t* qbuf = smem + C::kQ;
      const int sub = lane & 15, first_row = (warp - 2) * 2 + (lane >> 4);
      if constexpr (2 * R < C::kNs) {   // columns behind the pieces: zeros, once
        for (int i = threadIdx.x - 64; i < (C::kNs - 2 * R) * kHeadDim / 4; i += 64)
          for (int k = 0; k < C::kQBufs; ++k) reinterpret_cast<uint32_t*>(qbuf + k * C::kQBytes + 2 * R * kHeadDim)[i] = 0;
      }
      Block at = ctl.blocks[0];
      for (uint32_t part = 0;; ++part) {
        const uint32_t qb = part % C::kQBufs;
        if (part >= C::kQBufs &&
            !warp_wait(&ctl.q_empty[qb], ((part / C::kQBufs) & 1) ^ 1, P.wait_limit_ns, &ctl.abort)) {
          if (lane == 0) fail();
          break;
        }
        if (part > 0 && warp == 2 && lane == 0) ctl.blocks[qb] = at;
        uint4 x[R / 4];
#pragma unroll
        for (int k = 0; k < R / 4; ++k) {
          const int i = first_row + 4 * k, row = at.rb * R + i;
          const int t = row_token(row), hq = at.h * P.c.group + row - t * P.c.group;
          const long long tok = static_cast<long long>(at.r) * P.q_tokens + t;
          x[k] = make_uint4(0, 0, 0, 0);
          if (row < rows) x[k] = __ldg(reinterpret_cast<const uint4*>(P.q + tok * P.q_st + hq * P.q_sh) + sub);
          if (sub == 0) {
            ctl.seen[qb][i] = row < rows ? at.len - P.q_tokens + t + 1 : 0;
            ctl.out_at[qb][i] = row < rows ? tok * P.o_st + hq * P.o_sh : -1;
            ctl.lse_at[qb][i] = static_cast<int>(tok * P.c.hq) + hq;
          }
        }
#pragma unroll
        for (int k = 0; k < R / 4; ++k) {
          const int i = first_row + 4 * k;
          const uint32_t word[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
          uint32_t m = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) m = max(m, max(word[j] & 0x7fffu, (word[j] >> 16) & 0x7fffu));
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
          const bool finite = m < 0x7f80u;
          const float scale = __uint_as_float(piece_scale(m));
          uint32_t hi[2] = {0, 0}, lo[2] = {0, 0};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a = __uint_as_float(word[j] << 16) * scale, b = __uint_as_float(word[j] & 0xffff0000u) * scale;
            const uint32_t two = e4m3x2(a, b);
            const float2 f = e4m3x2_values(two);
            hi[j / 2] |= two << (16 * (j & 1));
            lo[j / 2] |= e4m3x2((a - f.x) * 16.f, (b - f.y) * 16.f) << (16 * (j & 1));
          }
          const auto put = [&](int n, const uint32_t* v) {
            *reinterpret_cast<uint2*>(qbuf + qb * C::kQBytes + n * kHeadDim + (((sub >> 1) ^ (n & 7)) << 4) +
                                      ((sub & 1) << 3)) = finite ? make_uint2(v[0], v[1]) : make_uint2(0, 0);
          };
          put(i, hi);
          put(R + i, lo);
          // a row with an infinity or a NaN: every logit NaN
          if (sub == 0) ctl.qs[qb][i] = finite ? P.alpha * __frcp_rn(scale) : __uint_as_float(0x7fc00000u);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.q_full[qb]);
        if (at.first + at.tiles >= x1) break;
        next_block(P, blocks, kTileKeys, at);
      }
    }
    // sequences without a token: their rows are zeros
    for (int r = blockIdx.x * 2 + warp - 2; r < P.n_seq; r += 2 * gridDim.x)
      if (seq_len(P, r) == 0)
        for (int i = 0; i < P.q_tokens * P.c.hq; ++i) {
          const int64_t tok = static_cast<int64_t>(r) * P.q_tokens + i / P.c.hq;
          reinterpret_cast<uint2*>(P.out + tok * P.o_st + (i % P.c.hq) * P.o_sh)[lane] = make_uint2(0, 0);
          if (P.lse && lane == 0) P.lse[tok * P.c.hq + i % P.c.hq] = -INFINITY;
        }
  } else if (works) {
    // ------------------------------------------------------------ softmax: a token, then a column, a thread
    const int half = H == 1 ? 0 : (warp >> 2) - 1, quad = warp & 3;
    const int tid = quad * 32 + lane, i0 = half * N;     // this thread's rows are i0 .. i0 + N - 1 of the block
    constexpr int kPartWords = N * (kHeadDim + 2);       // of a part: these rows, their maxima and sums
    const uint32_t my_lanes = static_cast<uint32_t>(quad) << 21;
    uint8_t* pbuf = smem + C::kP;
    uint32_t met = 0;
    // the 128 threads of these rows; what each wrote to shared memory before is seen behind it
    const auto meet_arrive = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.meet[half]);
    };
    const auto meet_wait = [&]() -> bool {
      return warp_wait(&ctl.meet[half], met++ & 1u, P.wait_limit_ns, &ctl.abort);
    };
    int len = 0, block0 = 0, block1 = 0;   // the part's sequence, its block's tiles of the line
    float unit = 0.f;                      // len_bits(len)
    const uint32_t n = x1 - x0;
    uint32_t part = 0;
    int splits = 0;
    struct End {
      bool whole, first;   // the part is its whole block; its block's first part
      int len;
      uint32_t part;
    };
    bool ok = true;
    float m = -INFINITY;                 // lane i: row i's maximum so far
    float l[N], acc[N];
    // adds tile `it`'s O^T
    const auto take = [&](uint32_t it) -> bool {
      if (!warp_wait(&ctl.o_full, it & 1, P.wait_limit_ns, &ctl.abort)) return false;
      tc_fence_after();
      if constexpr (H == 1) {
        float o[N == 4 ? 16 : 3 * N];
        if constexpr (N == 4) {
          tmem_ld16(tmem + C::kOCol + my_lanes, o);
        } else {
          static_assert(N == 8, "three loads of 8 columns");
#pragma unroll
          for (int k = 0; k < 3; ++k) tmem_ld8(tmem + C::kOCol + k * R + my_lanes, o + k * N);
        }
        tmem_wait_ld(o);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float y = fmaf(fmaf(o[2 * N + i], 0.0625f, o[N + i]), 0.0625f, o[i]);
          acc[i] = fmaf(y, ctl.back[it & 1][i0 + i], acc[i]);
        }
      } else {
        static_assert(N == 8, "a load of 8 columns a piece");
#pragma unroll
        for (int g = 0; g < N; g += 4) {   // (four rows at a time: 80 registers, and all together spill)
          float o[12];
#pragma unroll
          for (int k = 0; k < 3; ++k) tmem_ld4(tmem + C::kOCol + k * R + i0 + g + my_lanes, o + 4 * k);
          tmem_wait_ld(o);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = fmaf(fmaf(o[8 + i], 0.0625f, o[4 + i]), 0.0625f, o[i]);
            acc[g + i] = fmaf(y, ctl.back[it & 1][i0 + g + i], acc[g + i]);
          }
        }
      }
      return true;
    };
    const auto begin = [&]() {
#pragma unroll
      for (int i = 0; i < N; ++i) l[i] = acc[i] = 0.f;
      m = -INFINITY;
    };
    const auto rows_ready = [&]() -> bool {   // of a new part
      if (half == 0) ctl.nan_from[part % C::kQBufs][tid] = kNoNan;
      if (!warp_wait(&ctl.q_full[part % C::kQBufs], (part / C::kQBufs) & 1, P.wait_limit_ns, &ctl.abort)) return false;
      const Block& b = ctl.blocks[part % C::kQBufs];
      len = b.len;
      unit = len_bits(len);
      block0 = b.first;
      block1 = b.first + b.tiles;
      return true;
    };
    // The end of a part, first half: the row sums over the tokens' threads, each step halving the rows that a
    // lane has, then the lanes. They are everybody's behind the next meeting.
    const auto sum_rows = [&](uint32_t part) {
      int row = 0;
#pragma unroll
      for (int o = 16, c = N / 2; o > 0; o >>= 1, c >>= 1) {
        const bool up = lane & o;
        if (c > 0) {
#pragma unroll
          for (int i = 0; i < c; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, up ? l[i] : l[i + c], o);
            l[i] = (up ? l[i + c] : l[i]) + other;
          }
          row += up ? c : 0;
        } else {
          l[0] += __shfl_xor_sync(0xffffffffu, l[0], o);
        }
      }
      if (lane % (32 / N) == 0) ctl.sum[C::kQBufs > 2 ? part & 1 : 0][quad][i0 + row] = l[0];
    };
    // Second half, with the last tile's O^T added: the output, or the part for the join
    const auto emit = [&](const End& end) {
      const uint32_t qb = end.part % C::kQBufs;
      if (P.q_tokens > 1) {
        const int found = ctl.nan_from[qb][tid];
        const int from = found == kNoNan ? INT32_MAX : end.len - P.q_tokens + 1 + found;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (ctl.seen[qb][i0 + i] > from) acc[i] = __uint_as_float(0x7fc00000u);
      }
      float sum = 0.f;   // lane i: row i's
      if (lane < N)
      {
        const float(*warps)[R] = ctl.sum[C::kQBufs > 2 ? end.part & 1 : 0];
        sum = (warps[0][i0 + lane] + warps[1][i0 + lane]) + (warps[2][i0 + lane] + warps[3][i0 + lane]);
      }
      if (end.whole) {
        const float inv = sum == 0.f ? 0.f : __frcp_rn(sum);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const long long to = ctl.out_at[qb][i0 + i];
          const float f = __shfl_sync(0xffffffffu, inv, i);
          if (to >= 0) P.out[to + tid] = to_bf16(acc[i] * f);
        }
        if (P.lse && quad == 0 && lane < N && ctl.out_at[qb][i0 + lane] >= 0)
          P.lse[ctl.lse_at[qb][i0 + lane]] = log_sum(m + len_bits(end.len), sum);
      } else {
        // one of several parts of the block: left for the join. Slot 1 of the CTA is for a block's first part
        // (its own last one), slot 0 for a later one (its own first)
        float* dst = P.partial + (static_cast<int64_t>(blockIdx.x) * 2 + end.first) * kAttendPartWords +
                     half * kPartWords;
#pragma unroll
        for (int i = 0; i < N; ++i) __stcg(dst + i * kHeadDim + tid, acc[i]);
        if (quad == 0 && lane < N) {
          __stcg(dst + N * kHeadDim + lane, m);
          __stcg(dst + N * kHeadDim + N + lane, sum);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.q_empty[qb]);
    };
    // Where there are query rows for it the end of a part waits for its successor's first scores: the value
    // product passes meanwhile, and that tile's meeting is the sums' too.
    constexpr bool kLate = C::kQBufs > 2;
    begin();
    ok = rows_ready();
    bool due = false;       // the tile before ended a part (end), whose end is still to come
    End end = {};
    bool pending = false;   // the tile before is of this part and not added yet
    for (uint32_t it = 0; ok && it < n; ++it) {
      const int x = x0 + static_cast<int>(it);
      const uint32_t st = it % kVStages, qb = part % C::kQBufs;
      const int pos = (x - block0) * kTileKeys + tid;
      if (!warp_wait(&ctl.m_full[st], (it / kVStages) & 1, P.wait_limit_ns, &ctl.abort)) {
        ok = false;
        break;
      }
      const int pg = tid >> P.c.page_shift;
      const uint32_t have = ctl.pages[st];
      const bool held = (have >> pg & 1u) && pos < len;
      const float ks = ctl.ks[st][pg], lv = ctl.lvs[st][pg];
      const float vrest = held ? ctl.vs[st][pg] : 0.f, vtop = ctl.vtop[st];
      if (!warp_wait(&ctl.s_full[it & 1], (it >> 1) & 1, P.wait_limit_ns, &ctl.abort)) {
        ok = false;
        break;
      }
      tc_fence_after();
      float w[N];
      {
        float s[2 * N];
        const uint32_t from = tmem + (it & 1) * C::kNs + my_lanes;
        if constexpr (H == 1 && N == 4) {
          tmem_ld8(from, s);
        } else {
          tmem_ld8(from + i0, s);
          tmem_ld8(from + R + i0, s + N);
        }
        tmem_wait_ld(s);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = fmaf(s[N + i], 0.0625f, s[i]) * ctl.qs[qb][i0 + i] * ks;
      }
      const int tile0 = pos - tid, tile_end = tile0 + kTileKeys;
      const bool whole = have == (0xffu >> (kMostTilePages - (kTileKeys >> P.c.page_shift))) && tile_end <= len;
      const bool some = P.q_tokens > 1 && tile_end > len - P.q_tokens + 1;   // tokens that not all rows see
      if (!whole || some) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (!held || pos >= ctl.seen[qb][i0 + i]) w[i] = -INFINITY;
      }
      float* red = &ctl.red[it & 1][quad][i0];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float top = warp_max(w[i] + lv);
        if (lane == i) red[i] = top;
      }
      meet_arrive();
      // the tile before while the others arrive; its probabilities' buffer is free behind it
      if ((pending || due) && !take(it - 1)) {
        ok = false;
        break;
      }
      if (!meet_wait()) {
        ok = false;
        break;
      }
      if constexpr (kLate) {
        if (due) {
          emit(end);
          begin();
          due = false;
        }
      }
      if (lane < N) {   // lane i: row i's maximum
        const float top = fmaxf(fmaxf(ctl.red[it & 1][0][i0 + lane], ctl.red[it & 1][1][i0 + lane]),
                                fmaxf(ctl.red[it & 1][2][i0 + lane], ctl.red[it & 1][3][i0 + lane]));
        const float mn = fmaxf(m, top), to = mn == -INFINITY ? 0.f : mn, share = ex2(top - (to + unit));
        ctl.top[i0 + lane] = top == -INFINITY ? 0.f : top;
        ctl.kept[i0 + lane] = ex2(m - to);
        ctl.share[i0 + lane] = share;
        ctl.back[it & 1][i0 + lane] = share * vtop;
        m = mn;
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float p = ex2(w[i] - ctl.top[i0 + i]), kept = ctl.kept[i0 + i];
        acc[i] *= kept;   // (the tile before is in it; this one's product comes later)
        l[i] = fmaf(l[i], kept, p * ctl.share[i0 + i]);
        w[i] = p * vrest;
      }
      if (!whole || some) {   // (a scale that is NaN, of tokens that a row does not see)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (!held || pos >= ctl.seen[qb][i0 + i]) w[i] = 0.f;
      }
      // three e4m3 pieces of each probability: column k R + i of the token's row
      uint32_t out[up16(3 * N) / 4];
#pragma unroll
      for (int i = 0; i < up16(3 * N) / 4; ++i) out[i] = 0;
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        uint32_t a[3], b[3];
        e4m3_pieces(w[i], w[i + 1], a);
        e4m3_pieces(w[i + 2], w[i + 3], b);
#pragma unroll
        for (int k = 0; k < 3; ++k) out[(k * N + i) / 4] = __byte_perm(a[k], b[k], 0x5410);
      }
      if constexpr (H == 1) {
#pragma unroll
        for (int c = 0; c < C::kNp / 16; ++c)
          *reinterpret_cast<uint4*>(pbuf + c * (16 * kTileKeys) + tid * 16) =
              make_uint4(out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]);
      } else {
        static_assert(H == 1 || (R == 16 && N == 8), "a piece of 16 rows is 16 bytes, 8 a half");
#pragma unroll
        for (int k = 0; k < 3; ++k)
          *reinterpret_cast<uint2*>(pbuf + k * (16 * kTileKeys) + tid * 16 + half * 8) =
              make_uint2(out[2 * k], out[2 * k + 1]);
      }
      if (half == 0 && (!whole || some)) {
        if (!warp_wait(&ctl.v_full[st], (it / kVStages) & 1, P.wait_limit_ns, &ctl.abort)) {
          ok = false;
          break;
        }
        uint8_t* v = smem + C::kV + st * kTileBytes;
        if (!held) {
          // a probability of 0 does not undo a NaN: rows without a token are zeros
#pragma unroll
          for (int j = 0; j < kHeadDim / 16; ++j)   // (each lane from another 16 bytes on: no bank twice)
            reinterpret_cast<uint4*>(v + tid * kHeadDim)[(j + tid) % (kHeadDim / 16)] = make_uint4(0, 0, 0, 0);
        }
        if (some) {
          // nor may a NaN value that later rows see reach the earlier ones: it is taken out here, and given to
          // the rows that see it when the part ends. nan_from: the first position with a NaN in this
          // column, counted from the first one that not every row sees
          const int first = len - P.q_tokens + 1 - tile0, t0 = max(first, 0), t1 = min(len - tile0, kTileKeys);
          for (int t = t0; t < t1; ++t) {
            uint8_t* at8 = v + t * kHeadDim + (((tid >> 4) ^ (t & 7)) << 4) + (tid & 15);
            if ((have >> (t >> P.c.page_shift) & 1u) && (*at8 & 0x7f) == 0x7f) {
              const int f = t - first;
              if (f < ctl.nan_from[qb][tid]) ctl.nan_from[qb][tid] = static_cast<uint8_t>(f);
              *at8 = 0;
            }
          }
        }
      }
      fence_proxy_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.p_full);
      pending = !(x + 1 == x1 || x + 1 == block1);
      if (pending) continue;

      // ---------------------------------------------------------- the end of a part
      const End now = {block0 >= x0 && block1 <= x1, block0 >= x0, len, part};
      if (!now.whole) {
        if (tid == 0) ctl.split[splits] = ctl.blocks[qb];
        ++splits;
      }
      sum_rows(part);
      if constexpr (kLate) {
        end = now;
        due = true;
      } else {
        meet_arrive();
        if (!take(it) || !meet_wait()) {
          ok = false;
          break;
        }
        emit(now);
        begin();
      }
      if (x + 1 < x1) {
        ++part;
        ok = rows_ready();
      }
    }
    if (kLate && ok && due) {
      meet_arrive();
      ok = take(n - 1) && meet_wait();
      if (ok) emit(end);
    }

    // ------------------------------------------------------------ the join of blocks that several CTAs had parts of
    // Counted once this CTA's share is done (a fence under the loads of a running share takes 5 us), by the
    // first CTA that has a part of the block; the CTA that counts last joins.
    allow_next_kernel();
    if (ok && splits > 0) {
      int w0 = 0, w1 = 0;
      if (tid < splits) ctl.cuts.parts(ctl.split[tid], &w0, &w1);
      meet_arrive();
      ok = meet_wait();
      if (ok && tid < splits)
        ctl.last[2 * half + tid] =
            inc_acq_rel_gpu(P.arrive + w0 * H + half, static_cast<unsigned>(w1 - w0)) == static_cast<unsigned>(w1 - w0)
                ? w1 - w0 + 1 : 0;
      if (tid < splits) ctl.split_cta[2 * half + tid] = w0;
      if (ok) {
        meet_arrive();
        ok = meet_wait();
      }
      // The parts are brought into the tiles' memory (nothing else uses it now: this CTA's tiles are done),
      // kBatch at a time; then a warp a row, four columns a lane, every sum in the order of the tokens.
      constexpr int kBatch = C::kQ / H / (kPartWords * 4);
      float* buf = reinterpret_cast<float*>(smem) + half * (C::kQ / H / 4);
      uint32_t copied = 0;
      for (int k = 0; ok && k < splits; ++k) {
        const int parts = ctl.last[2 * half + k];
        if (parts == 0) continue;
        const Block b = ctl.split[k];
        const int first = ctl.split_cta[2 * half + k];
        float top[N / 4], sum[N / 4];
        float4 a4[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          top[i] = -INFINITY;
          sum[i] = 0.f;
          a4[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        for (int p0 = 0; ok && p0 < parts; p0 += kBatch) {
          const int count = min(parts - p0, kBatch);
          if (quad == 0) {
            fence_proxy_async();   // the others' stores, and our reads of the batch before, then the copies
            if (lane == 0) mbar_arrive_expect_tx(&ctl.joined[half], count * (kPartWords * 4));
            __syncwarp();
            for (int j = lane; j < count; j += 32)   // part p: slot 0 of CTA first + p, of the first one slot 1
              bulk_load(buf + j * kPartWords,
                        P.partial + (static_cast<int64_t>(first + p0 + j) * 2 + (p0 + j == 0)) * kAttendPartWords +
                            half * kPartWords,
                        kPartWords * 4, &ctl.joined[half]);
          }
          ok = warp_wait(&ctl.joined[half], copied & 1u, P.wait_limit_ns, &ctl.abort);
          if (!ok) {
            if (lane == 0) mbar_wait(&ctl.joined[half], copied & 1u, P.wait_limit_ns, &ctl.never);   // (in flight)
            break;
          }
          ++copied;
#pragma unroll
          for (int i = 0; i < N / 4; ++i) {
            const float* row = buf + (quad + 4 * i) * kHeadDim;
            const float* stats = buf + N * kHeadDim + quad + 4 * i;
            float mn = top[i];
            for (int j = lane; j < count; j += 32) mn = fmaxf(mn, stats[j * kPartWords]);
            mn = warp_max(mn);
            const float ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(top[i] - ref);
            top[i] = mn;
            sum[i] *= f0;
            a4[i].x *= f0, a4[i].y *= f0, a4[i].z *= f0, a4[i].w *= f0;
#pragma unroll 2
            for (int j = 0; j < count; ++j) {
              const float g = ex2(stats[j * kPartWords] - ref);
              const float4 o = reinterpret_cast<const float4*>(row + j * kPartWords)[lane];
              sum[i] = fmaf(stats[j * kPartWords + N], g, sum[i]);
              a4[i].x = fmaf(o.x, g, a4[i].x);
              a4[i].y = fmaf(o.y, g, a4[i].y);
              a4[i].z = fmaf(o.z, g, a4[i].z);
              a4[i].w = fmaf(o.w, g, a4[i].w);
            }
          }
          meet_arrive();
          ok = meet_wait();   // the batch has been read
        }
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          const int row = b.rb * R + i0 + quad + 4 * i;
          if (row >= rows) break;
          const int t = row_token(row), hq = b.h * P.c.group + row - t * P.c.group;
          const int64_t tok = static_cast<int64_t>(b.r) * P.q_tokens + t;
          const float inv = sum[i] == 0.f ? 0.f : __frcp_rn(sum[i]);
          uint2 v;
          v.x = to_bf16(a4[i].x * inv) | static_cast<uint32_t>(to_bf16(a4[i].y * inv)) << 16;
          v.y = to_bf16(a4[i].z * inv) | static_cast<uint32_t>(to_bf16(a4[i].w * inv)) << 16;
          reinterpret_cast<uint2*>(P.out + tok * P.o_st + hq * P.o_sh)[lane] = v;
          if (P.lse && lane == 0) P.lse[tok * P.c.hq + hq] = log_sum(top[i] + len_bits(b.len), sum[i]);
        }
      }
    }
    if (!ok && lane == 0) fail();
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, C::kTmemCols);
  }
}

template <int R, int H>
cudaError_t attend_rows(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  constexpr size_t smem = attend_smem<R, H>();
  auto* fn = cache_attend_kernel<R, H>;
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  // no more CTAs than there can be tiles
  const int64_t blocks = (p.q_tokens * p.c.group + R - 1) / R;
  const int64_t tiles = ((static_cast<int64_t>(p.c.max_pages) << p.c.page_shift) + kTileKeys - 1) / kTileKeys;
  const int64_t most = static_cast<int64_t>(kAttendCtas) * c.sms;
  const int64_t want = tiles >= most ? most : tiles * p.n_seq * p.c.heads * blocks;
  return launch_after_previous(fn, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(ACfg<R, H>::kThreads),
                               smem, stream, c.tm_k, c.tm_v, p);
}

}  // namespace

cudaError_t launch_cache_attend(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  const int rows = p.q_tokens * p.c.group;
  if (rows <= 4) return attend_rows<4, 1>(c, p, stream);
  if (rows <= 8) return attend_rows<8, 1>(c, p, stream);
  return attend_rows<16, 2>(c, p, stream);
}

}  // namespace kve
