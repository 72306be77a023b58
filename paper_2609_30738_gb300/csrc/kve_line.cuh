// How the attention over a paged cache is cut: the tiles of all (sequence, head, row block)s in one line, an even
// share of it for every CTA, whatever the lengths, which are read on the GPU. Blocks, cuts and the walk over them are those of the 8-bit
// cache's attention too; that has line_share's steps in a body of its own, around its tensor memory's allocation (kve_attend.cu), and
// what Cuts::parts says has to hold for both.
#pragma once

#include "kve_internal.h"
#include "kve_ptx.cuh"

namespace kve {

// A (sequence, head, row block): the rows of one row block over one sequence's tiles, `first` their first in
// the line of all tiles.
struct Block {
  int r, h, rb, len, tiles, first;
  int index;   // its number among all blocks that have tiles
};

// No more CTAs take part than have kLeastUnits units each, or a block.
constexpr int kLeastUnits = 4;

// A part costs about kPart tiles besides its own (its query rows, the latency at its two ends, its output), so a block
// counts as its tiles and kPart more units, and the units are dealt evenly: CTA w's raw cut is floor(units * w /
// ctas). A cut that would leave fewer than `least` tiles of a block on one of its sides moves to that end of the block: a
// join costs more than those tiles do.
template <int kPart>
struct Cuts {
  int each, rest, ctas, units, least;
  uint32_t inverse;   // of ctas, 2^32 / ctas rounded up: exact for the products below ctas^2 that it divides
  __device__ __forceinline__ void set(int n, int w) {
    units = n;
    ctas = w;
    each = n / w;
    rest = n - each * w;
    least = each <= 8 ? 4 : 2;
    inverse = 0xffffffffu / static_cast<uint32_t>(w) + 1u;   // (for one CTA 0, and rest is 0)
  }
  __device__ __forceinline__ int raw(int w) const {
    return each * w + static_cast<int>(__umulhi(static_cast<uint32_t>(rest * w), inverse));
  }
  // the first w with raw(w) >= u
  __device__ __forceinline__ int from(int u) const {
    int w = min(max(static_cast<int>(static_cast<float>(u) * static_cast<float>(ctas) / static_cast<float>(units)), 0), ctas);
    while (w > 0 && raw(w - 1) >= u) --w;
    while (w < ctas && raw(w) < u) ++w;
    return w;
  }
  // CTAs [*w0, *w1] have the parts of block b
  __device__ __forceinline__ void parts(const Block& b, int* w0, int* w1) const {
    const int a = b.first + (b.index + 1) * kPart;   // its tile 0 in units
    *w0 = from(a + least) - 1;
    *w1 = from(a + b.tiles - least + 1) - 1;
  }
};

__device__ __forceinline__ int seq_len(const AttendParams& P, int r) {
  return min(max(__ldg(P.lens + r), 0), P.c.max_pages << P.c.page_shift);
}

// The block behind b in the line; a tile follows, so a sequence that is not empty does.
__device__ __forceinline__ void next_block(const AttendParams& P, int blocks, int tile, Block& b) {
  b.first += b.tiles;
  ++b.index;
  if (++b.rb < blocks) return;
  b.rb = 0;
  if (++b.h < P.c.heads) return;
  b.h = 0;
  do {
    b.len = seq_len(P, ++b.r);
    b.tiles = (b.len + tile - 1) / tile;
  } while (b.tiles == 0);
}

// log2 of the unit in which a row's sums over tokens are held where they could leave fp32, 2^-len_bits(len) of themselves: then a
// sum passes the largest value as little as the average does (values of 2e38 would leave fp32 from two of them on).
__device__ __forceinline__ float len_bits(int len) { return static_cast<float>(32 - __clz(len - 1)); }   // (1: 0)

template <int kWarps>
struct LineCtl {
  int2 sums[kWarps];   // tiles, sequences that have some
  int ends[2];         // this CTA's tiles of the line
  Block first;         // the block of its first tile
};

// This CTA's share of the line, in ctl, and the cuts. Every thread of the kWarps warps comes here (and meets the others
// behind it). A length outside 0 .. max_pages * P, or a line of 2^30 tiles, sets the error word.
template <int kWarps, int kPart>
__device__ __forceinline__ void line_share(const AttendParams& P, int blocks, int tile, LineCtl<kWarps>& ctl,
                                           Cuts<kPart>& cuts) {
  constexpr int kThreads = 32 * kWarps;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // a run of sequences a thread
  const int cap = P.c.max_pages << P.c.page_shift;
  const int per = (P.n_seq + kThreads - 1) / kThreads;
  const int s0 = min(static_cast<int>(threadIdx.x) * per, P.n_seq), s1 = min(s0 + per, P.n_seq);
  int mine = 0, filled = 0;   // tiles of one block each (2^30: too many), sequences that have some
  bool bad = false;
  for (int r = s0; r < s1; ++r) {
    const int len = __ldg(P.lens + r);
    bad |= len < 0 || len > cap;
    mine = min(mine + (min(max(len, 0), cap) + tile - 1) / tile, 1 << 30);
    filled += len > 0;
  }
  __syncwarp();
  int front = mine, front_filled = filled;   // up to and with this thread's sequences
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, front, o), y = __shfl_up_sync(0xffffffffu, front_filled, o);
    if (lane >= o) {
      front = min(front + x, 1 << 30);
      front_filled += y;
    }
  }
  if (lane == 31) ctl.sums[warp] = make_int2(front, front_filled);
  if (threadIdx.x == 0) ctl.ends[0] = ctl.ends[1] = 0;
  bad = __syncthreads_or(bad);
  int all_tiles = 0, all_filled = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
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
  const int per_seq = P.c.heads * blocks;   // blocks of a sequence
  const long long all_units = (static_cast<long long>(all_tiles) + static_cast<long long>(all_filled) * kPart) * per_seq;
  const bool too_long = all_tiles >= 1 << 30 || all_units >= 1 << 30;
  if ((bad || too_long) && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(P.err, kErrCheck);
  const int units = too_long ? 0 : static_cast<int>(all_units);
  cuts.set(units, max(min(max(units / kLeastUnits, all_filled * per_seq), static_cast<int>(gridDim.x)), 1));
  if (units > 0 && static_cast<int>(blockIdx.x) < cuts.ctas) {
    // the thread that holds a cut's sequence says which tile of the line it is
    const int c0 = cuts.raw(blockIdx.x), c1 = cuts.raw(blockIdx.x + 1);
    int at = front * per_seq, index = front_filled * per_seq;   // tiles, blocks in front
    if (threadIdx.x == 0 && c1 == units) ctl.ends[1] = all_tiles * per_seq;
    for (int r = s0; r < s1; ++r) {
      const int len = seq_len(P, r), tiles = (len + tile - 1) / tile;
      if (tiles == 0) continue;
      const int unit = at + index * kPart, size = tiles + kPart;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = (e ? c1 : c0) - unit;
        if (c < 0 || c >= size * per_seq) continue;
        int b = c / size, j = c - b * size - kPart;   // block of the sequence, tiles in front of the cut
        if (j < cuts.least) {
          j = 0;
        } else if (tiles - j < cuts.least) {
          j = 0;
          ++b;   // (a block's end is the next one's start)
        }
        ctl.ends[e] = at + b * tiles + j;
        if (e == 0) {
          const int h = b / blocks;
          // (b = per_seq: behind the sequence, found below)
          ctl.first = {r, h, b - h * blocks, len, tiles, at + b * tiles, index + b};
        }
      }
      at += tiles * per_seq;
      index += per_seq;
    }
  }
  __syncthreads();
  if (ctl.ends[0] < ctl.ends[1] && ctl.first.h == P.c.heads) {   // (for all threads) the next sequence that has tiles
    __syncthreads();
    if (threadIdx.x == 0) {
      Block f = ctl.first;
      f.h = f.rb = 0;
      do {
        f.len = seq_len(P, ++f.r);
        f.tiles = (f.len + tile - 1) / tile;
      } while (f.tiles == 0);
      ctl.first = f;
    }
    __syncthreads();
  }
}

// One output row: a quarter of the average of v (four columns a lane), the log2 of the largest p, sum p in units of that.
template <class RowToken>
__device__ __forceinline__ void emit_row(const AttendParams& P, const Block& b, int row, int rows, RowToken row_token,
                                         const float4& a, float top, float sum, int lane) {
  if (row >= rows) return;
  const int t = row_token(row), hq = b.h * P.c.group + row - t * P.c.group;
  const int64_t tok = static_cast<int64_t>(b.r) * P.q_tokens + t;
  const auto pair = [&](float x, float y) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(y * 4.f), "f"(x * 4.f));
    return d;
  };
  reinterpret_cast<uint2*>(P.out + tok * P.o_st + hq * P.o_sh)[lane] = make_uint2(pair(a.x, a.y), pair(a.z, a.w));
  if (P.lse && lane == 0)
    P.lse[tok * P.c.hq + hq] = sum == 0.f ? -INFINITY : (top + lg2(sum)) * 0.69314718056f;
}

}  // namespace kve
