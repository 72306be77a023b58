// The paged 8-bit cache: its C entry points, and the kernels that keep its tables and write its
// pages (the attention that reads them is in kve_attend.cu).
//
// A page holds P tokens of every cache head: e4m3 codes and one power-of-two scale per (page, head).
// For the rows that share a scale and their largest finite magnitude a,
//   need(a) = 2^e, the smallest e >= -126 with a <= 448 * 2^e,   code = RN_e4m3(x / scale).
// Division by a power of two is exact, so a code is rounded once, and a page whose scale grows by 2^k
// keeps RN(x / 2^e) / 2^k = RN(x / 2^(e+k)) for every code that stays normal.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>

#include "kve_internal.h"
#include "kve_ptx.cuh"
#include "kve_rotary.cuh"

namespace kve {
namespace {

// ---------------------------------------------------------------- tables and slots

constexpr int kPagesThreads = 1024;
constexpr int64_t kPagesCtas = 152;   // one an SM: twice as many took 3.2 us more on those prompts, half twice the time
constexpr int kPagesWarps = kPagesThreads / 32;
static_assert(kPagesWarps == 32, "a lane a sequence of the CTA");

// A sequence that changes: lengths, its first place in the ring, its slots (or null), its table row.
struct Grown {
  int32_t a, b, ring;
  int32_t* out;
  int32_t* row;
};

// The warp's sum of x < 2^50 (in two parts whose sums fit 32 bits).
__device__ __forceinline__ long long warp_sum(long long x) {
  const uint32_t lo = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(x) & 0xffffffu);
  const uint32_t hi = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(x >> 24));
  return (static_cast<long long>(hi) << 24) + lo;
}

__device__ __forceinline__ int ring_at(int head, long long i, int n) {
  // head < n and i <= n (checked before any use)
  long long p = head + i;
  if (p >= n) p -= n;
  if (p >= n) p -= n;
  return static_cast<int>(p);
}

// A CTA has 32 sequences, a warp each for their places in the ring and in their layer's slots; their pages, in
// chunks of 32 (a lane a page), are one line that the warps share, so that one long sequence is no warp's
// alone. A chunk's pages are read in one access, while the chunk before is written, and its slots leave from
// registers, four at a time: new pages cost their 8 bytes and slots their 4. Before that every CTA sums the pages
// and tokens that each layer takes and gives (a warp a layer), so that all agree whether the call can be done
// before one of them writes. Where the call changes its inputs in place (lens_out, ring_out), the CTA that finishes
// reading last does that.
//
// A decode step (512 sequences, one new token each) is bound by latency: two reads of 8 bytes a sequence from L2
// and the chain length -> ring entry -> table: 4.8 us. A wave of prompts is bound by the slots' write: 48 of 500 to
// 32768 tokens in 32 layers (P = 16, 67 MB) 17.6 us, 56% of a copy's 6780 GB/s, of which 5.5 are the decode step's
// latencies; 201 MB of slots at P = 64 40 us. Slots one at a time took 19.0 and 45.8, four without the read ahead 19.5
// and 40.6.
//
// Every CTA reads all lengths, so there is never more than one an SM: with more than 32 sequences for each (kMany) a CTA
// takes several groups of 32 after one sum. A sequence's place costs a sum over its layer's sequences in front, so the
// step stays quadratic in those of one layer: decode steps of 32 layers x 256 sequences 10.8 us, 32 x 1024 45 (72 with a
// CTA for each 32), 64 x 1024 94 (205).
template <bool kMany>
__global__ void __launch_bounds__(kPagesThreads) cache_pages_kernel(const __grid_constant__ PagesParams P) {
  wait_previous_kernel();
  __shared__ long long layer_sum[3][kMaxLayers];   // pages taken, pages given, new tokens
  __shared__ Grown grown[kPagesWarps];
  __shared__ int chunks_of[kPagesWarps];
  __shared__ uint32_t bad_word, last_word;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int S = P.c.max_seqs, layers = P.c.num_layers, n = layers * S;
  const int shift = P.c.page_shift, page_mask = P.c.page - 1;
  const int cap = P.c.max_pages << shift;
  const int head = __ldg(P.ring_in), count = __ldg(P.ring_in + 1), np = P.c.num_pages;
  if (threadIdx.x == 0) bad_word = 0;
  __syncthreads();
  bool bad = false;
  const auto sum_of = [&](const int32_t* from, const int32_t* to, int m, long long (&sum)[3]) {
    uint32_t taken = 0, given = 0;   // (below 2^27 pages a sequence, 32 of them a lane)
    long long tokens = 0;
    for (int i = lane; i < m; i += 32) {
      const int a = __ldg(from + i), b = __ldg(to + i);
      bad |= a < 0 || b < 0 || a > cap || b > cap;
      const int d = ((b + page_mask) >> shift) - ((a + page_mask) >> shift);
      taken += max(d, 0);
      given += max(-d, 0);
      tokens += max(b - a, 0);
    }
    sum[0] = warp_sum(taken);
    sum[1] = warp_sum(given);
    sum[2] = P.slots ? warp_sum(tokens) : 0;
  };
#pragma unroll 4
  for (int l = warp; l < layers; l += kPagesWarps) {
    long long sum[3];
    sum_of(P.from + l * S, P.to + l * S, S, sum);
    if (lane < 3) layer_sum[lane][l] = lane == 0 ? sum[0] : lane == 1 ? sum[1] : sum[2];
  }
  if (bad) bad_word = 1;
  __syncthreads();
  int seq = blockIdx.x * kPagesWarps + warp;
  int layer = seq < n ? seq / S : layers - 1, r = seq - layer * S;
  long long taken = 0, given = 0, at = 0, back = 0;
  bool too_many = false;
  for (int l = lane; l < layers; l += 32) {
    const long long x = layer_sum[0][l], y = layer_sum[1][l];
    taken += x;
    given += y;
    at += l < layer ? x : 0;
    back += l < layer ? y : 0;
    too_many |= P.slots && layer_sum[2][l] > P.slot_stride;
  }
  taken = warp_sum(taken);
  given = warp_sum(given);
  bad = bad_word || __any_sync(0xffffffffu, too_many) || head < 0 || head >= np || count < 0 || count > np ||
        count + given > np;
  const bool ok = !bad && taken <= count;
  for (;;) {
    // this warp's sequence: its chunks of 32 pages, its place in the ring and in its layer's slots
    int chunks = 0;
    if (seq < n && ok) {
      const int a = __ldg(P.from + seq), b = __ldg(P.to + seq);
      const int have = (a + page_mask) >> shift, need = (b + page_mask) >> shift;
      // from the page of the first new token on, or the released ones
      chunks = b > a ? (need - (a >> shift) + 31) >> 5 : (have - need + 31) >> 5;
      if (chunks > 0) {
        long long before[3];
        sum_of(P.from + layer * S, P.to + layer * S, r, before);
        at = warp_sum(at) + before[0];
        back = warp_sum(back) + before[1];
        if (lane == 0) {
          grown[warp] = {a, b, ring_at(head, b > a ? at : count + back, np),
                         b > a && P.slots ? P.slots + layer * P.slot_stride + before[2] : nullptr,
                         P.table + static_cast<int64_t>(seq) * P.c.max_pages};
        }
      }
    }
    if (lane == 0) chunks_of[warp] = chunks;
    __syncthreads();
    // all chunks of this CTA's sequences in one line, dealt to its warps (and those of the other blockIdx.y)
    int last = chunks_of[lane];
  #pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, last, o);
      if (lane >= o) last += x;
    }
    const int all = __shfl_sync(0xffffffffu, last, 31);
    // the page of a chunk's lane is read while the chunk before it is written
    struct Chunk {
      int w, c, page;   // its sequence, its number there, this lane's page (-1: none)
    };
    const auto read = [&](int q) {
      Chunk k;
      k.w = __popc(__ballot_sync(0xffffffffu, last <= q)) & 31;   // the sequence whose chunk it is
      const int before = __shfl_sync(0xffffffffu, last, max(k.w - 1, 0));
      k.c = q - (k.w > 0 ? before : 0);
      k.page = -1;
      if (q >= all) return k;
      const Grown& s = grown[k.w];
      const int have = (s.a + page_mask) >> shift, need = (s.b + page_mask) >> shift;
      if (s.b > s.a) {
        const int j = (s.a >> shift) + 32 * k.c + lane;
        if (j < have)
          k.page = s.row[j];
        else if (j < need)
          k.page = P.free_pages[ring_at(s.ring, j - have, np)];
      } else {
        const int j = need + 32 * k.c + lane;
        if (j < have) k.page = s.row[j];
      }
      return k;
    };
    const int first = blockIdx.y * kPagesWarps + warp, step = kPagesWarps * gridDim.y;
    Chunk next = read(first);
    for (int q = first; q < all; q += step) {
      const Chunk now = next;
      if (q + step < all) next = read(q + step);
      const Grown s = grown[now.w];
      const int c = now.c, page = now.page;
      const int have = (s.a + page_mask) >> shift, need = (s.b + page_mask) >> shift;
      if (s.b > s.a) {
        const int j0 = (s.a >> shift) + 32 * c, j = j0 + lane;
        if (j >= have && j < need) s.row[j] = page;
        const int base = page >= 0 && page < np ? page << shift : -1;
        const bool outside = __any_sync(0xffffffffu, j < need && base < 0);   // a page outside the pool
        if (outside && lane == 0) atomicOr(P.err, kErrCheck);
        if (!s.out) continue;
        // slots [begin, end) of the chunk, counted from its first page
        const int begin = max(s.a - (j0 << shift), 0), end = min(s.b - (j0 << shift), 32 << shift), len = end - begin;
        int32_t* const to = s.out + ((j0 << shift) + begin - s.a);
        if (outside) {
          // its tokens get no slot
  #pragma unroll 1
          for (int i = 0; i < len; i += 32) {
            const int k = begin + i + lane;
            const int from = __shfl_sync(0xffffffffu, base, k >> shift);
            if (i + lane < len) to[i + lane] = from < 0 ? -1 : from + (k & page_mask);
          }
          continue;
        }
        // up to the first multiple of 16 bytes and behind the last one by slot, in between four at a time
        const int front = min(static_cast<int>(-(reinterpret_cast<uintptr_t>(to) >> 2) & 3), len);
        const int quads = (len - front) >> 2, rest = (len - front) & 3;
        {
          const int i = lane < 16 ? lane : len - 32 + lane, k = begin + i;
          const int from = __shfl_sync(0xffffffffu, base, k >> shift);
          if (lane < front || lane >= 32 - rest) to[i] = from + (k & page_mask);
        }
  #pragma unroll 2
        for (int i = 0; i < quads; i += 32) {
          const int q = front + 4 * (i + lane), k = begin + q, off = k & page_mask;
          const int x = __shfl_sync(0xffffffffu, base, k >> shift) + off;
          const int y = __shfl_sync(0xffffffffu, base, (k + 3) >> shift) + off - P.c.page;   // of those on the next page
          if (i + lane < quads)
            *reinterpret_cast<int4*>(to + q) =
                make_int4(x, (off + 1 < P.c.page ? x : y) + 1, (off + 2 < P.c.page ? x : y) + 2,
                          (off + 3 < P.c.page ? x : y) + 3);
        }
      } else {
        const int j = need + 32 * c + lane;
        if (j < have) P.free_pages[ring_at(s.ring, j - need, np)] = page;
      }
    }
    if (seq < n) {
      if (P.slots && r == S - 1) {
        // behind the layer's new tokens (from its start where nothing was done)
        int32_t* out = P.slots + layer * P.slot_stride;
        for (int64_t i = (ok ? layer_sum[2][layer] : 0) + lane + 32 * blockIdx.y; i < P.slot_stride; i += 32 * gridDim.y)
          out[i] = -1;
      }
    }
    if (!P.in_place && seq < n && lane == 0 && blockIdx.y == 0) P.lens_out[seq] = ok ? P.to[seq] : P.from[seq];
    if constexpr (!kMany) break;
    seq += gridDim.x * kPagesWarps;
    if (seq - warp >= n) break;
    layer = seq < n ? seq / S : layers - 1;
    r = seq - layer * S;
    at = back = 0;
    for (int l = lane; l < layer; l += 32) {
      at += layer_sum[0][l];
      back += layer_sum[1][l];
    }
    __syncthreads();   // (the group before is written)
  }
  if (!P.in_place) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
      P.ring_out[0] = ok ? ring_at(head, taken, np) : head;
      P.ring_out[1] = ok ? static_cast<int>(count - taken + given) : count;
      *P.refused = ok ? 0 : 1;
      if (!ok) atomicOr(P.err, bad ? kErrCheck : kErrPages);
    }
    allow_next_kernel();
    return;
  }
  // the last CTA moves the state on
  __syncthreads();
  const uint32_t ctas = gridDim.x * gridDim.y;
  if (threadIdx.x == 0) last_word = inc_acq_rel_gpu(P.done, ctas - 1) == ctas - 1;
  __syncthreads();
  allow_next_kernel();
  if (!last_word) return;
  const int32_t* now = ok ? P.to : P.from;
  if (P.lens_out != now)
    for (int i = threadIdx.x; i < n; i += kPagesThreads) P.lens_out[i] = now[i];
  if (threadIdx.x == 0) {
    P.ring_out[0] = ok ? ring_at(head, taken, np) : head;
    P.ring_out[1] = ok ? static_cast<int>(count - taken + given) : count;
    *P.refused = ok ? 0 : 1;
    if (!ok) atomicOr(P.err, bad ? kErrCheck : kErrPages);
  }
}

__global__ void cache_reset_kernel(int32_t* free_pages, int32_t* ring, int n) {
  wait_previous_kernel();
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) free_pages[i] = i;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    ring[0] = 0;
    ring[1] = n;
  }
}

// ---------------------------------------------------------------- rows in 8 bits

// A run (new rows of one page and head, of keys or of values) is written by a team of P / kGroupRows groups
// of 16 lanes; group g holds page rows kGroupRows g .. in registers, 8 elements of each row a lane, from the
// load of a row to the store of its codes: bf16 is read once and codes are written once, whatever P.
//
// Bound by HBM: 256 bytes read and 128 written a row. A team's loads are all in flight before its maximum is
// known and its stores wait for that, so the overlap is between CTAs, and small ones do best: with one team
// of 128 or 256 threads a CTA (P = 64, 128) or four smaller ones, 16 prompts at a budget of 509 in 8 layers
// (387 MB) take 68.5 us, 83% of a copy's 6780 GB/s, and 24k prompt tokens (146 MB) 27.6 us, 78%; with 256 threads
// for P = 64 73.6 and 29.8, with 16 rows a group 119 and 30.5, with 4 rows 92 and 42.6.
constexpr int kGroupRows = 8;
template <int kPage>
constexpr int kTeamThreads = kPage / kGroupRows * 16;   // a warp at least
template <int kPage>
constexpr int kRowThreads = kTeamThreads<kPage> >= 128 ? kTeamThreads<kPage> : 4 * kTeamThreads<kPage>;

// The larger magnitudes of two bf16 pairs; NaN counts only where both are.
__device__ __forceinline__ uint32_t max_abs(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("{\n .reg .b32 x, y;\n abs.bf16x2 x, %1;\n abs.bf16x2 y, %2;\n max.bf16x2 %0, x, y;\n}" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The pair x without its infinities and NaN.
__device__ __forceinline__ uint32_t finite_only(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0x0000ffffu;
  return x;
}

// need(a) as fp32 bits for the magnitude with bf16 bits a (finite): a = (1 + f/128) 2^(x-127), and
// 448 = 1.75 * 2^8, so e = x - 127 - 8, one more where the fraction passes 1.75 (f > 96).
__device__ __forceinline__ uint32_t need_bits(uint32_t a) {
  const int e = static_cast<int>(a >> 7) - 8 + ((a & 0x7fu) > 96u ? 1 : 0);
  return static_cast<uint32_t>(max(e, 1)) << 23;
}

__device__ __forceinline__ uint2 row_codes(const uint4& x, float inv) {
  const auto two = [&](uint32_t p) {
    return e4m3x2(__uint_as_float(p << 16) * inv, __uint_as_float(p & 0xffff0000u) * inv);
  };
  return make_uint2(two(x.x) | two(x.y) << 16, two(x.z) | two(x.w) << 16);
}

// Two e4m3 codes times f, as e4m3 codes again.
__device__ __forceinline__ uint32_t scaled_codes(uint32_t two, float f) {
  const float2 x = e4m3x2_values(two);
  return e4m3x2(x.x * f, x.y * f);
}

// Waits for the other groups of this thread's team.
template <int kPage>
__device__ __forceinline__ void team_sync() {
  constexpr int kTeam = kTeamThreads<kPage>;
  if constexpr (kTeam == kRowThreads<kPage>)
    __syncthreads();
  else if constexpr (kTeam > 32)
    named_bar_sync(1 + threadIdx.x / kTeam, kTeam);
  else
    __syncwarp();
}

// The largest finite magnitude of a group's rows (8 elements of each a lane), as bf16 bits, in all its lanes.
__device__ __forceinline__ uint32_t group_max(const uint4 (&x)[kGroupRows], uint32_t lanes) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kGroupRows; ++i) m = max_abs(m, max_abs(max_abs(x[i].x, x[i].y), max_abs(x[i].z, x[i].w)));
  if ((m & 0x7f80u) == 0x7f80u || (m & 0x7f800000u) == 0x7f800000u) {
    // an infinity or nothing but NaN among them (rare): the finite ones alone
    m = 0;
#pragma unroll
    for (int i = 0; i < kGroupRows; ++i)
      m = max_abs(m, max_abs(max_abs(finite_only(x[i].x), finite_only(x[i].y)),
                             max_abs(finite_only(x[i].z), finite_only(x[i].w))));
  }
  m = max(m & 0xffffu, m >> 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(lanes, m, o));
  return m;
}

// Rows row0 .. end - 1 of a page to a scale that is 1 / f of theirs (their rounding again only where they become
// subnormal), four in flight: beside the rows to be written there is no room for more.
__device__ __forceinline__ void shrink_rows(uint8_t* codes, int row0, int end, float f, int lane) {
  constexpr int kBatch = 4;
#pragma unroll 1
  for (; row0 < end; row0 += kBatch) {
    uint2 c[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (row0 + i < end) c[i] = reinterpret_cast<const uint2*>(codes + (row0 + i) * kHeadDim)[lane];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (row0 + i < end) {
        c[i].x = scaled_codes(c[i].x & 0xffffu, f) | scaled_codes(c[i].x >> 16, f) << 16;
        c[i].y = scaled_codes(c[i].y & 0xffffu, f) | scaled_codes(c[i].y >> 16, f) << 16;
        reinterpret_cast<uint2*>(codes + (row0 + i) * kHeadDim)[lane] = c[i];
      }
  }
}

// Where a lane's 8 elements lie in a row: side by side, or as two pieces of 4, a and b.
struct SideBySide {
  int lane;
  __device__ __forceinline__ uint4 load(const uint16_t* row) const { return __ldg(reinterpret_cast<const uint4*>(row) + lane); }
  __device__ __forceinline__ void store(uint8_t* row, uint2 codes) const { reinterpret_cast<uint2*>(row)[lane] = codes; }
};
struct TwoPieces {
  int a, b;
  __device__ __forceinline__ uint4 load(const uint16_t* row) const {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(row) + a), y = __ldg(reinterpret_cast<const uint2*>(row) + b);
    return make_uint4(x.x, x.y, y.x, y.y);
  }
  __device__ __forceinline__ void store(uint8_t* row, uint2 codes) const {
    reinterpret_cast<uint32_t*>(row)[a] = codes.x;
    reinterpret_cast<uint32_t*>(row)[b] = codes.y;
  }
};

// Writes rows [off, off + n) of a page (codes and scale of one head); x[i] holds this lane's 8
// elements of page row kGroupRows g + i, zero outside the run. Every thread of the team comes here.
template <int kPage, class Where>
__device__ __forceinline__ void write_run(const uint4 (&x)[kGroupRows], int off, int n, uint8_t* codes, float* scale,
                                          uint32_t* team_max, const Where& where) {
  constexpr int kGroups = kPage / kGroupRows;
  const int lane = threadIdx.x & 15, g = (threadIdx.x / 16) % kGroups;
  uint32_t m = group_max(x, threadIdx.x & 16 ? 0xffff0000u : 0x0000ffffu);
  // the page's scale is read before it is written: every group reads, then all meet
  const float held = off > 0 ? *scale : 0.f;
  if (lane == 0) team_max[g] = m;
  team_sync<kPage>();
#pragma unroll
  for (int i = 0; i < kGroups; ++i) m = max(m, team_max[i]);
  const float s = fmaxf(held, __uint_as_float(need_bits(m)));
  const float inv = __frcp_rn(s);   // exact: a power of two
  if (s > held && off > 0) shrink_rows(codes, g * kGroupRows, min((g + 1) * kGroupRows, off), held * inv, lane);
#pragma unroll
  for (int i = 0; i < kGroupRows; ++i) {
    const int row = g * kGroupRows + i;
    if (static_cast<uint32_t>(row - off) < static_cast<uint32_t>(n)) where.store(codes + row * kHeadDim, row_codes(x[i], inv));
  }
  if (g == 0 && lane == 0) *scale = s;
}

// The same by one group, for a run of at most kGroupRows rows: x[i] is page row off + i, zero behind the run.
template <class Where>
__device__ __forceinline__ void write_short_run(const uint4 (&x)[kGroupRows], int off, int n, uint8_t* codes,
                                                float* scale, const Where& where) {
  const int lane = threadIdx.x & 15;
  const uint32_t lanes = threadIdx.x & 16 ? 0xffff0000u : 0x0000ffffu;
  const float held = off > 0 ? *scale : 0.f;
  const uint32_t m = group_max(x, lanes);
  __syncwarp(lanes);   // all have read the scale
  const float s = fmaxf(held, __uint_as_float(need_bits(m)));
  const float inv = __frcp_rn(s);
  if (s > held) shrink_rows(codes, 0, off, held * inv, lane);
#pragma unroll
  for (int i = 0; i < kGroupRows; ++i)
    if (i < n) where.store(codes + (off + i) * kHeadDim, row_codes(x[i], inv));
  if (lane == 0) *scale = s;
}

// Step 4 into the cache. A team takes page j of a unit, keys or values (the two alternate).
template <int kPage>
__global__ void __launch_bounds__(kRowThreads<kPage>) cache_gather_kernel(const __grid_constant__ CacheGatherParams P) {
  wait_previous_kernel();   // the indices come from the selection launched before
  constexpr int kTeam = kTeamThreads<kPage>, kGroups = kPage / kGroupRows, kTeams = kRowThreads<kPage> / kTeam;
  __shared__ uint32_t team_max[kTeams][kGroups];
  const int team = threadIdx.x / kTeam, lane = threadIdx.x & 15, g = (threadIdx.x / 16) % kGroups;
  const uint32_t item = blockIdx.x * kTeams + team;   // (below 2^31)
  const uint32_t pages = item >> 1, unit = pages / P.unit_pages;
  if (unit >= P.g.g.n_units) return;   // the whole team
  const bool values = item & 1;
  const int j = static_cast<int>(pages - unit * P.unit_pages);
  const UnitInfo u = unit_info(P.g.g, unit);
  const int W = P.g.g.window, Lc = u.L - W;
  const int m = min(P.g.layer_budget[u.layer], Lc);
  const int n = min(m + W - j * kPage, kPage);
  if (n <= 0) return;
  const int seq = u.layer * P.c.max_seqs + P.first_seq + u.r;
  const int page = __ldg(P.table + static_cast<int64_t>(seq) * P.c.max_pages + j);
  const bool refused = __ldg(P.refused) != 0;   // the table's pages may be other sequences' by now
  // the positions of this group's rows: lane i looks row i's up
  const int row = j * kPage + g * kGroupRows + (lane & (kGroupRows - 1));
  int src = -1;
  bool outside = false;
  if (row < m) {
    src = __ldg(P.g.indices + static_cast<int64_t>(unit) * P.g.budget + row);
    outside = src < 0 || src >= Lc;   // never read outside the unit: a row of zeros, and the status tells
    if (outside) src = -1;
  } else if (row < m + W) {
    src = Lc + (row - m);
  }
  if (refused) return;
  if (outside) atomicOr(P.err, kErrCheck);
  if (page < 0 || page >= P.c.num_pages) {
    if (g == 0 && lane == 0) atomicOr(P.err, kErrCheck);
    return;
  }
  const uint16_t* from = values ? P.g.v + u.v_off : P.g.k + u.k_off;
  const int64_t st = values ? P.g.g.v_st : P.g.g.k_st;
  const uint32_t lanes = threadIdx.x & 16 ? 0xffff0000u : 0x0000ffffu;
  uint4 x[kGroupRows];
#pragma unroll
  for (int i = 0; i < kGroupRows; ++i) {
    const int s = __shfl_sync(lanes, src, i, 16);
    x[i] = make_uint4(0, 0, 0, 0);
    if (s >= 0) x[i] = __ldg(reinterpret_cast<const uint4*>(from + s * st) + lane);
  }
  const int64_t block = static_cast<int64_t>(page) * P.c.heads + u.h;
  write_run<kPage>(x, 0, n, (values ? P.c.v : P.c.k) + block * (kPage * kHeadDim),
                   (values ? P.c.v_scale : P.c.k_scale) + block, team_max[team], SideBySide{lane});
  allow_next_kernel();
}

// New tokens by slot. A team takes `block` consecutive tokens (P, or P / 8) of one head, keys or values, and writes
// the runs that start among them: one after the other by the whole team where they are long (a prompt's, a page
// each), all at once by a group each where they are short (a decode step's tokens, drafts). Every warp lists the
// runs by itself from the slots, a lane a token: a token continues a run where its slot is the one behind its
// predecessor's on the same page. Runs of up to kGroupRows rows fit a group's registers and are short.
//
// A block of P / 8 tokens gives a small call more teams, one of P tokens a large one fewer scans (P = 64, P / 8
// against P, us): 256 sequences x 1 token 3.3 and 11.1, 1000 x 1 7.3 and 11.5, 1000 x 2 9.3 and 8.2, 1000 x 8 29.1
// and 12.6; one prompt of 512 3.4 and 2.9, of 1024 4.9 and 3.2, of 4096 11.8 and 5.3. P = 16: 3.5 and 13.4, 7.3 and
// 13.9, 12.7 and 8.8, 28.4 and 13.3; 3.9 and 3.1, 5.3 and 3.4, 12.5 and 5.8. So P for more than 1024 tokens: the
// steps of up to 1024 sequences keep the small blocks, and prompts of 512 to 1024 tokens pay for it (what decides is
// the length of the runs, which the host does not know). Decode steps of 16 and 256 sequences (8 heads) take
// 2.6 and 3.4 us, mostly the launch and three loads in a row (slots, scale, rows); a team a token with the runs found
// from 16 lanes took 2.9 and 4.15. Drafts, 1000 x 8 tokens at any offset, 49 MB, take 14.4 us where HBM would take
// 7.3: 2000 teams of 8 runs, of which 1216 fit at once, are two rounds of that chain.
constexpr int64_t kStoreBlockTokens = 1024;

// Threads an SM: the rotating append's have the turns of their rows beside the rows. (512, 640, 768, 896, 1024: 24k tokens 107.4, 99.2,
// 96.5, 97.8 and 102.6 us, 2000 tokens 11.6, 11.0, 10.4, 11.7 and 12.7, 16 tokens 2.6, 2.8, 2.8, 3.0 and 3.2.)
template <class Params>
constexpr int kStoreThreads = std::is_same_v<Params, CacheAppendParams> ? 768 : 1024;

__device__ __forceinline__ const CacheStoreParams& rows_of(const CacheStoreParams& p) { return p; }
__device__ __forceinline__ const CacheStoreParams& rows_of(const CacheAppendParams& p) { return p.s; }

// Of a row that turns, each of 16 lanes has both elements of four pairs, as its two pieces: no lane waits for another's, and no
// turn is computed twice in a row.
struct LaneTurns {
  uint2 turn[4];
  bool turns;
  __device__ __forceinline__ TwoPieces set(const RotaryTable& r, int lane) {
    turns = 4 * lane < r.pairs;
#pragma unroll
    for (int i = 0; i < 4; ++i) turn[i] = turn_at(r, 4 * lane + i);   // (of 64)
    if (!r.interleaved && turns) return {lane, lane + (r.pairs >> 2)};
    return {2 * lane, 2 * lane + 1};
  }
};

// Turns the rows x[i] of tokens token0 + i (those with row0 + i in 0 .. n - 1; 16 lanes have a row), rounded to bf16 as a
// rotation by itself would leave them. pos: in lane i, token i's position.
__device__ __forceinline__ void turn_rows(uint4 (&x)[kGroupRows], const RotaryTable& r, int pos, int row0, int n,
                                          const LaneTurns& turn) {
  const uint32_t lanes = threadIdx.x & 16 ? 0xffff0000u : 0x0000ffffu;
#pragma unroll
  for (int i = 0; i < kGroupRows; ++i) {
    if (static_cast<uint32_t>(row0 + i) >= static_cast<uint32_t>(n)) continue;   // (all 16 lanes)
    const int p = __shfl_sync(lanes, pos, i, 16);
    if (!turn.turns) continue;
    float2 cs[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) cs[k] = turn_of(turn.turn[k], r.amplitude, p);
    if (r.interleaved) {
      turn_neighbours(x[i], cs);
    } else {
      uint32_t a[2] = {x[i].x, x[i].y}, b[2] = {x[i].z, x[i].w};
      turn_halves(a, b, cs);
      x[i] = make_uint4(a[0], a[1], b[0], b[1]);
    }
  }
}

// With parameters of the rotating append the CTAs behind the first row_ctas turn the queries, and those turn the keys on their
// way: they start first because they take longer (as the last: 2000 tokens 14.8 us for 11.7, 400 x 8 23.1 for 20.1, 24k 102.6
// for 101.9; evenly between the others 13.6, 24.5 and 112, all at the time). 24k tokens with 32 query heads (537 MB) take 96.5 us of
// 80.3 at a copy's rate, 6000 without their queries 16.8 of 9.2: every head's rows compute their turns. Pages of 16 and 32 spill 76
// bytes: 24k tokens 103 us, 1000 x 8 40.4 for 36.7, 16 3.3 for 2.9. (With elements side by side, the
// pairs' halves exchanged by shuffles, 100.9 and 18.9; turns kept in shared memory for four heads one after the other 114.9, for two
// 120.) One body with the plain store as a kernel of its own: as a function of both it spilled three times as much.
template <int kPage, class Params>
__global__ void __launch_bounds__(kRowThreads<kPage>, kStoreThreads<Params> / kRowThreads<kPage>)
cache_store_kernel(const __grid_constant__ Params A, uint32_t row_ctas) {
  constexpr bool kTurn = std::is_same_v<Params, CacheAppendParams>;
  wait_previous_kernel();
  if constexpr (kTurn) {
    __shared__ __align__(16) float2 turns[kTurnTokens * kMaxPairs];
    if (blockIdx.x >= row_ctas) {
      rotate_tile<kRowThreads<kPage>, 4>(A.turn, blockIdx.x - row_ctas, turns);
      allow_next_kernel();
      return;
    }
  }
  const CacheStoreParams& P = rows_of(A);
  constexpr int kTeam = kTeamThreads<kPage>, kGroups = kPage / kGroupRows, kTeams = kRowThreads<kPage> / kTeam;
  constexpr int kWords = kPage / 16;   // of 32 tokens: a block of at most P and the run that leaves it
  __shared__ uint32_t team_max[kTeams][kGroups];
  __shared__ uint32_t goes_on[kRowThreads<kPage> / 32][kWords];
  __shared__ uint16_t runs[kRowThreads<kPage> / 32][kPage];   // first token << 8 | tokens: long, from the end short
  const int team = threadIdx.x / kTeam, lane = threadIdx.x & 15, g = (threadIdx.x / 16) % kGroups;
  const int warp = threadIdx.x >> 5, lane32 = threadIdx.x & 31;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kTeams + team;
  const int H = P.c.heads;
  const int64_t first = item / (2 * H) * P.block;
  if (first >= P.n_tokens) return;   // the whole team
  const int hv = static_cast<int>(item % (2 * H)), h = hv >> 1;
  const bool values = hv & 1;
  const uint16_t* from = (values ? P.v + h * P.v_sh : P.k + h * P.k_sh);
  const int64_t st = values ? P.v_st : P.k_st;
  uint8_t* const codes = values ? P.c.v : P.c.k;
  float* const scales = values ? P.c.v_scale : P.c.k_scale;
  const int32_t* slots = P.slots + first;
  const int64_t left = P.n_tokens - first;
  LaneTurns turn;
  std::conditional_t<kTurn, TwoPieces, SideBySide> where = {};
  if constexpr (kTurn) {
    where = {2 * lane, 2 * lane + 1};
    if (!values) where = turn.set(A.turn.r, lane);
  } else {
    where = {lane};
  }
  // the slots of the block and of what a run can reach behind it
  int longs = 0, shorts = 0;
  {
    int here[kWords];
#pragma unroll
    for (int c = 0; c < kWords; ++c) here[c] = 32 * c + lane32 < left ? __ldg(slots + 32 * c + lane32) : -1;
    int before = first > 0 ? __ldg(slots - 1) : -1;
    constexpr int kFirst = kPage > 32 ? kPage / 32 : 1;   // words of the block
    uint32_t begins[kFirst];
#pragma unroll
    for (int c = 0; c < kWords; ++c) {
      int prev = __shfl_up_sync(0xffffffffu, here[c], 1);
      if (lane32 == 0) prev = before;
      before = __shfl_sync(0xffffffffu, here[c], 31);
      const bool on = here[c] >= 0 && prev >= 0 && here[c] - prev == 1 && (here[c] & (kPage - 1)) != 0;
      const uint32_t word = __ballot_sync(0xffffffffu, on);
      if (lane32 == 0) goes_on[warp][c] = word;
      const uint32_t b = __ballot_sync(0xffffffffu, here[c] >= 0 && !on && 32 * c + lane32 < P.block);
      if (c < kFirst) begins[c] = b;
    }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < kFirst; ++c) {
      if (begins[c] == 0) continue;
      const bool mine = begins[c] >> lane32 & 1u;
      const int t = 32 * c + lane32;
      int n = 1;   // tokens of the run that starts here: those that go on without a gap
      if (mine)
        for (int p = t + 1; p < 32 * kWords;) {
          const uint32_t gap = ~(goes_on[warp][p >> 5] >> (p & 31));
          const int ones = min(gap ? __ffs(gap) - 1 : 32, 32 - (p & 31));
          n += ones;
          p += ones;
          if ((p & 31) != 0 || ones == 0) break;
        }
      const bool is_long = mine && n > kGroupRows;
      const uint32_t l = __ballot_sync(0xffffffffu, is_long), b = begins[c] & ~l, below = (1u << lane32) - 1u;
      if (is_long) runs[warp][longs + __popc(l & below)] = static_cast<uint16_t>(t << 8 | n);
      if (mine && !is_long) runs[warp][kPage - 1 - shorts - __popc(b & below)] = static_cast<uint16_t>(t << 8 | n);
      longs += __popc(l);
      shorts += __popc(b);
    }
    __syncwarp();
  }
  const int limit = P.c.num_pages * kPage;   // (below 2^31)
  for (int k = 0; k < longs + shorts;) {
    const bool whole_team = k < longs;
    const int at = whole_team ? k : kPage - 1 - (k - longs) - g;   // (short ones: this group's)
    if (whole_team) {
      ++k;
    } else {
      const bool none = k - longs + g >= shorts;
      k += kGroups;
      if (none) continue;
    }
    const int t = runs[warp][at] >> 8, n = runs[warp][at] & 255;
    const int slot = __ldg(slots + t);
    if (slot >= limit) {
      if (lane == 0) atomicOr(P.err, kErrCheck);
      continue;
    }
    const int off = slot & (kPage - 1);
    const int64_t block = static_cast<int64_t>(slot / kPage) * H + h;
    const int row0 = whole_team ? g * kGroupRows - off : 0;   // the run's row in x[0]
    uint4 x[kGroupRows];
    int pos = 0;
    if constexpr (kTurn) {
      if (!values && static_cast<uint32_t>(row0 + lane) < static_cast<uint32_t>(n) && lane < kGroupRows)
        pos = __ldg(A.turn.positions + first + t + row0 + lane);
    }
#pragma unroll
    for (int i = 0; i < kGroupRows; ++i) {
      x[i] = make_uint4(0, 0, 0, 0);
      if (static_cast<uint32_t>(row0 + i) < static_cast<uint32_t>(n))
        x[i] = where.load(from + (first + t + row0 + i) * st);
    }
    if constexpr (kTurn) {
      if (!values) turn_rows(x, A.turn.r, pos, row0, n, turn);
    }
    if (whole_team) {
      write_run<kPage>(x, off, n, codes + block * (kPage * kHeadDim), scales + block, team_max[team], where);
      team_sync<kPage>();   // team_max and the scale before the next run
    } else {
      write_short_run(x, off, n, codes + block * (kPage * kHeadDim), scales + block, where);
    }
  }
  allow_next_kernel();
}

template <int kPage>
int64_t store_ctas(const CacheStoreParams& p) {
  constexpr int kTeams = kRowThreads<kPage> / kTeamThreads<kPage>;
  const int64_t items = (p.n_tokens + p.block - 1) / p.block * 2 * p.c.heads;
  return (items + kTeams - 1) / kTeams;
}

template <int kPage>
cudaError_t store_paged(const CacheStoreParams& p, cudaStream_t stream) {
  return launch_after_previous(cache_store_kernel<kPage, CacheStoreParams>, dim3(static_cast<unsigned>(store_ctas<kPage>(p))),
                               dim3(kRowThreads<kPage>), 0, stream, p, 0u);
}

template <int kPage>
cudaError_t append_paged(const CacheAppendParams& params, cudaStream_t stream) {
  CacheAppendParams p = params;
  const int64_t turn_tiles = p.turn.heads > 0 ? cut_rotate<kRowThreads<kPage>>(p.turn) : 0, row_ctas = store_ctas<kPage>(p.s);
  return launch_after_previous(cache_store_kernel<kPage, CacheAppendParams>, dim3(static_cast<unsigned>(row_ctas + turn_tiles)),
                               dim3(kRowThreads<kPage>), 0, stream, p, static_cast<uint32_t>(row_ctas));
}

template <int kPage>
cudaError_t gather_paged(const CacheGatherParams& p, cudaStream_t stream) {
  constexpr int kTeams = kRowThreads<kPage> / kTeamThreads<kPage>;
  const int64_t items = p.g.g.n_units * p.unit_pages * 2;
  return launch_after_previous(cache_gather_kernel<kPage>, dim3(static_cast<unsigned>((items + kTeams - 1) / kTeams)),
                               dim3(kRowThreads<kPage>), 0, stream, p);
}

}  // namespace

cudaError_t launch_cache_pages(const PagesParams& p, cudaStream_t stream) {
  const int n = p.c.num_layers * p.c.max_seqs;
  const int64_t groups = (n + kPagesWarps - 1) / kPagesWarps, x = std::min(groups, kPagesCtas);
  // CTAs that share 32 sequences: what their slots (or table rows) ask for, one CTA an SM in all
  const int64_t tokens = p.slots ? (p.slot_stride + p.c.max_seqs - 1) / p.c.max_seqs : int64_t(p.c.max_pages) << p.c.page_shift;
  int64_t y = (tokens >> p.c.page_shift) / 32;
  const int64_t most = x < kPagesCtas ? kPagesCtas / x : 1;
  y = y > most ? most : y;
  return launch_after_previous(groups > x ? cache_pages_kernel<true> : cache_pages_kernel<false>, dim3(static_cast<unsigned>(x), static_cast<unsigned>(y < 1 ? 1 : y)),
                               dim3(kPagesThreads), 0, stream, p);
}

cudaError_t launch_cache_reset(const kve_cache& c, int32_t* free_pages, int32_t* ring, cudaStream_t stream) {
  const int blocks = (c.geo.num_pages + 255) / 256;
  return launch_after_previous(cache_reset_kernel, dim3(blocks < 304 ? blocks : 304), dim3(256), 0, stream,
                               free_pages, ring, c.geo.num_pages);
}

cudaError_t launch_cache_gather(const CacheGatherParams& p, cudaStream_t stream) {
  switch (p.c.page) {
    case 16: return gather_paged<16>(p, stream);
    case 32: return gather_paged<32>(p, stream);
    case 64: return gather_paged<64>(p, stream);
    default: return gather_paged<128>(p, stream);
  }
}

static int store_block(const CacheStoreParams& p) {
  return p.n_tokens > kStoreBlockTokens ? p.c.page : p.c.page / kGroupRows;
}

cudaError_t launch_cache_append(const CacheAppendParams& params, cudaStream_t stream) {
  CacheAppendParams p = params;
  p.s.block = store_block(p.s);
  switch (p.s.c.page) {
    case 16: return append_paged<16>(p, stream);
    case 32: return append_paged<32>(p, stream);
    case 64: return append_paged<64>(p, stream);
    default: return append_paged<128>(p, stream);
  }
}

cudaError_t launch_cache_store(const CacheStoreParams& params, cudaStream_t stream) {
  CacheStoreParams p = params;
  p.block = store_block(p);
  switch (p.c.page) {
    case 16: return store_paged<16>(p, stream);
    case 32: return store_paged<32>(p, stream);
    case 64: return store_paged<64>(p, stream);
    default: return store_paged<128>(p, stream);
  }
}

bool row_strides(const int64_t* given, int64_t heads, int64_t* token, int64_t* head) {
  *token = given ? given[0] : heads * kHeadDim;
  *head = given ? given[1] : kHeadDim;
  for (const int64_t s : {*token, *head})
    if (s < 0 || s % 8 != 0 || s >= (int64_t(1) << 37)) return false;
  return true;
}

// Tokens outside heads, or heads outside tokens.
bool rows_apart(int64_t tokens, int64_t token, int64_t heads, int64_t head) {
  const auto apart = [](int64_t inner, int64_t count, int64_t outer, int64_t outer_count) {
    return (count <= 1 || inner >= kHeadDim) &&
           (outer_count <= 1 || outer >= (count > 0 ? (count - 1) * inner : 0) + kHeadDim);
  };
  return apart(head, heads, token, tokens) || apart(token, tokens, head, heads);
}

int place_of(const void* p) {
  cudaPointerAttributes at;
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return kUnknown;
  }
  return at.type == cudaMemoryTypeDevice ? at.device : at.type == cudaMemoryTypeHost ? kHostMemory : kUnknown;
}

}  // namespace kve

namespace {

using kve::kHeadDim;
using kve::kHostMemory;
using kve::place_of;
using kve::row_strides;

constexpr uint64_t kWaitNs = 2000000000ull;   // every device-side wait, 2 s

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The call's device is the buffers' device.
bool on_device(const kve_cache* c) {
  if (c->device < 0) return true;
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == c->device;
}

// A cache of `bits`, with the given scales (8) or numbers of the rows (4).
kve_status create_cache(const kve_cache_config* cfg, int bits, uint8_t* k, uint8_t* v, void* k_scale, void* v_scale,
                        kve_cache** cache_out, size_t* workspace_bytes) {
  if (!cfg || !k || !v || !k_scale || !v_scale || !cache_out) return KVE_EINVAL;
  *cache_out = nullptr;
  const kve_cache_config& c = *cfg;
  if (c.num_layers < 1 || c.num_layers > kve::kMaxLayers || c.head_dim != kHeadDim) return KVE_EINVAL;
  if (c.num_kv_heads < 1 || c.num_kv_heads > kve::kMaxCacheHeads || c.num_q_heads < c.num_kv_heads ||
      c.num_q_heads % c.num_kv_heads || c.num_q_heads / c.num_kv_heads > kve::kMaxRows)
    return KVE_EINVAL;
  if (c.page_tokens != 16 && c.page_tokens != 32 && c.page_tokens != 64 && c.page_tokens != 128) return KVE_EINVAL;
  if (c.num_pages < 1 || c.max_pages < 1 || c.max_pages > c.num_pages || c.max_seqs < 1 ||
      c.max_seqs > kve::kMaxCacheSeqs)
    return KVE_EINVAL;
  // rows of the pool are 32-bit TMA coordinates
  if (static_cast<int64_t>(c.num_pages) * c.page_tokens >= (int64_t(1) << 31) / c.num_kv_heads) return KVE_EINVAL;
  if (!aligned(k, 128) || !aligned(v, 128) || !aligned(k_scale, 16) || !aligned(v_scale, 16)) return KVE_EINVAL;
  // the kernels follow all four: device memory of one device
  const int device = place_of(k);
  if (device == kHostMemory) return KVE_EINVAL;
  for (const void* p : {static_cast<const void*>(v), static_cast<const void*>(k_scale), static_cast<const void*>(v_scale)})
    if (place_of(p) != device) return KVE_EINVAL;
  kve_cache* h = new (std::nothrow) kve_cache;
  if (!h) return KVE_ENOMEM;
  std::memset(h, 0, sizeof(*h));
  kve::CacheGeometry& g = h->geo;
  g.num_layers = c.num_layers;
  g.hq = c.num_q_heads;
  g.heads = c.num_kv_heads;
  g.group = c.num_q_heads / c.num_kv_heads;
  g.page = c.page_tokens;
  for (g.page_shift = 0; (1 << g.page_shift) < g.page;) ++g.page_shift;
  g.num_pages = c.num_pages;
  g.max_pages = c.max_pages;
  g.max_seqs = c.max_seqs;
  g.k = k;
  g.v = v;
  h->bits = bits;
  if (bits == 8) {
    g.k_scale = static_cast<float*>(k_scale);
    g.v_scale = static_cast<float*>(v_scale);
  } else {
    g.k_param = static_cast<uint32_t*>(k_scale);
    g.v_param = static_cast<uint32_t*>(v_scale);
  }
  h->device = device;
  int dev = device, sms = 0;
  if ((dev < 0 && cudaGetDevice(&dev) != cudaSuccess) ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    sms = 152;   // no device visible: size for a full GB300
  }
  h->sms = sms;
  kve::CacheWsLayout& w = h->ws;
  w.err = 0;
  w.pages_done = 64;
  w.refused = 128;
  w.arrive = 256;
  static_assert(kve::kAttend4PartWords == kve::kAttendPartWords, "one size for both");
  const size_t workers = static_cast<size_t>(bits == 8 ? kve::kAttendCtas : kve::kAttend4Ctas) * sms;
  w.clear_end = align_up(w.arrive + sizeof(uint32_t) * 2 * workers, 256);
  w.partial = w.clear_end;
  w.total = align_up(w.partial + workers * 2 * kve::kAttendPartWords * sizeof(float), 256);
  h->maps = bits == 8 && kve::encode_pages(&h->tm_k, k, g) && kve::encode_pages(&h->tm_v, v, g);
  if (workspace_bytes) *workspace_bytes = w.total;
  *cache_out = h;
  return KVE_OK;
}

uint32_t* word(void* ws, size_t at) { return reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(ws) + at); }

// The checks and parameters of a store, with or without a rotation.
kve_status store_params(const kve_cache* cache, const uint16_t* k_new, const uint16_t* v_new, const int64_t* k_strides,
                        const int64_t* v_strides, const int32_t* slots, int64_t n_tokens, void* ws,
                        kve::CacheStoreParams* p) {
  if (!cache || n_tokens < 0 || n_tokens > INT32_MAX / (2 * kve::kMaxCacheHeads) || !ws || !aligned(ws, 256))
    return KVE_EINVAL;
  if (n_tokens > 0 && (!k_new || !v_new || !slots)) return KVE_EINVAL;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(slots, 4)) return KVE_EINVAL;
  std::memset(p, 0, sizeof(*p));
  p->c = cache->geo;
  if (!row_strides(k_strides, p->c.heads, &p->k_st, &p->k_sh) || !row_strides(v_strides, p->c.heads, &p->v_st, &p->v_sh))
    return KVE_EINVAL;
  if (!on_device(cache)) return KVE_EINVAL;
  p->k = k_new;
  p->v = v_new;
  p->slots = slots;
  p->n_tokens = n_tokens;
  p->err = word(ws, cache->ws.err);
  return KVE_OK;
}

}  // namespace

extern "C" {

kve_status kv_evict_cache_create(const kve_cache_config* cfg, uint8_t* k, uint8_t* v, float* k_scale,
                                 float* v_scale, kve_cache** cache_out, size_t* workspace_bytes) {
  return create_cache(cfg, 8, k, v, k_scale, v_scale, cache_out, workspace_bytes);
}

kve_status kv_evict_cache4_create(const kve_cache_config* cfg, uint8_t* k, uint8_t* v, uint16_t* k_param,
                                  uint16_t* v_param, kve_cache** cache_out, size_t* workspace_bytes) {
  return create_cache(cfg, 4, k, v, k_param, v_param, cache_out, workspace_bytes);
}

void kv_evict_cache_destroy(kve_cache* cache) { delete cache; }

kve_status kv_evict_cache_reset(const kve_cache* cache, int32_t* free_pages, int32_t* ring, void* ws, void* stream) {
  if (!cache || !ws || !aligned(ws, 256) || !free_pages != !ring) return KVE_EINVAL;
  if (free_pages && (!aligned(free_pages, 4) || !aligned(ring, 4))) return KVE_EINVAL;
  if (!on_device(cache)) return KVE_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cudaMemsetAsync(ws, 0, cache->ws.clear_end, st) != cudaSuccess) return KVE_ECUDA;
  if (free_pages && kve::launch_cache_reset(*cache, free_pages, ring, st) != cudaSuccess) return KVE_ECUDA;
  return KVE_OK;
}

kve_status kv_evict_cache_pages(const kve_cache* cache, const int32_t* lens_from, const int32_t* lens_to,
                                int32_t* table, int32_t* free_pages, const int32_t* ring_in, int32_t* ring_out,
                                int32_t* lens_out, int32_t* slots, int64_t slot_stride, void* ws, void* stream) {
  if (!cache || !lens_from || !lens_to || !table || !free_pages || !ring_in || !ring_out || !lens_out || !ws)
    return KVE_EINVAL;
  for (const void* p : {static_cast<const void*>(lens_from), static_cast<const void*>(lens_to),
                        static_cast<const void*>(table), static_cast<const void*>(free_pages),
                        static_cast<const void*>(ring_in), static_cast<const void*>(ring_out),
                        static_cast<const void*>(lens_out), static_cast<const void*>(slots)})
    if (!aligned(p, 4)) return KVE_EINVAL;
  if (!aligned(ws, 256) || slot_stride < 0 || (slots && slot_stride > INT32_MAX)) return KVE_EINVAL;
  if (!on_device(cache)) return KVE_EINVAL;
  kve::PagesParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = cache->geo;
  p.from = lens_from;
  p.to = lens_to;
  p.table = table;
  p.free_pages = free_pages;
  p.ring_in = ring_in;
  p.ring_out = ring_out;
  p.lens_out = lens_out;
  p.slots = slots;
  p.slot_stride = slot_stride;
  p.err = word(ws, cache->ws.err);
  p.done = word(ws, cache->ws.pages_done);
  p.refused = word(ws, cache->ws.refused);
  p.in_place = lens_out == lens_from || lens_out == lens_to || ring_out == ring_in;
  return kve::launch_cache_pages(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KVE_OK : KVE_ECUDA;
}

kve_status kv_evict_cache_gather(const kve_cache* cache, const kve_plan* plan, const uint16_t* k, const uint16_t* v,
                                 const int32_t* indices, int32_t first_seq, const int32_t* table, void* ws,
                                 void* stream) {
  if (!cache || !plan || !k || !v || !indices || !table || !ws) return KVE_EINVAL;
  const kve::Geometry& g = plan->geo;
  const kve::CacheGeometry& c = cache->geo;
  if (g.num_layers != c.num_layers || g.uheads != c.heads || first_seq < 0 || first_seq > c.max_seqs - g.n_req)
    return KVE_EINVAL;
  // the most rows that a unit of this plan keeps
  int64_t rows = 0;
  for (int l = 0; l < g.num_layers; ++l)
    for (int r = 0; r < g.n_req; ++r)
      rows = std::max<int64_t>(rows, std::min(plan->layer_budget[l], g.req_len[r] - g.window) + g.window);
  const int64_t pages = (rows + c.page - 1) / c.page;
  if (pages > c.max_pages) return KVE_EINVAL;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(indices, 4) || !aligned(table, 4) || !aligned(ws, 256))
    return KVE_EINVAL;
  // teams of one launch
  if (g.n_units * pages * 2 >= (int64_t(1) << 31)) return KVE_EINVAL;
  if (!kve::readable_source(k) || !kve::readable_source(v) || !on_device(cache)) return KVE_EINVAL;
  kve::CacheGatherParams p;
  std::memset(&p, 0, sizeof(p));
  p.g.g = g;
  p.g.budget = plan->cfg.budget;
  for (int l = 0; l < g.num_layers; ++l) p.g.layer_budget[l] = plan->layer_budget[l];
  p.g.k = k;
  p.g.v = v;
  p.g.indices = indices;
  p.c = c;
  p.table = table;
  p.first_seq = first_seq;
  p.unit_pages = static_cast<int32_t>(pages);
  p.refused = word(ws, cache->ws.refused);
  p.err = word(ws, cache->ws.err);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->bits == 4 ? kve::launch_cache4_gather(p, st) : kve::launch_cache_gather(p, st);
  return e == cudaSuccess ? KVE_OK : KVE_ECUDA;
}

kve_status kv_evict_cache_store(const kve_cache* cache, const uint16_t* k_new, const uint16_t* v_new,
                                const int64_t* k_strides, const int64_t* v_strides, const int32_t* slots,
                                int64_t n_tokens, void* ws, void* stream) {
  kve::CacheStoreParams p;
  const kve_status bad = store_params(cache, k_new, v_new, k_strides, v_strides, slots, n_tokens, ws, &p);
  if (bad != KVE_OK || n_tokens == 0) return bad;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->bits == 4 ? kve::launch_cache4_store(p, st) : kve::launch_cache_store(p, st);
  return e == cudaSuccess ? KVE_OK : KVE_ECUDA;
}

kve_status kv_evict_cache_append(const kve_cache* cache, const kve_rotary* rotary, const int32_t* positions,
                                 const uint16_t* q, const int64_t* q_strides, uint16_t* q_out,
                                 const int64_t* q_out_strides, const uint16_t* k_new, const uint16_t* v_new,
                                 const int64_t* k_strides, const int64_t* v_strides, const int32_t* slots,
                                 int64_t n_tokens, void* ws, void* stream) {
  kve::CacheAppendParams p;
  if (!rotary || !q != !q_out || (n_tokens > 0 && !positions) || !aligned(positions, 4)) return KVE_EINVAL;
  const kve_status bad = store_params(cache, k_new, v_new, k_strides, v_strides, slots, n_tokens, ws, &p.s);
  if (bad != KVE_OK) return bad;
  std::memset(&p.turn, 0, sizeof(p.turn));
  if (q) {
    const int32_t hq = cache->geo.hq;
    if (!aligned(q, 16) || !aligned(q_out, 16) || n_tokens >= (int64_t(1) << 31) / hq) return KVE_EINVAL;
    if (!row_strides(q_strides, hq, &p.turn.x_st, &p.turn.x_sh) ||
        !row_strides(q_out_strides, hq, &p.turn.o_st, &p.turn.o_sh) ||
        !kve::rows_apart(n_tokens, p.turn.o_st, hq, p.turn.o_sh))
      return KVE_EINVAL;
    if (q == q_out && (p.turn.x_st != p.turn.o_st || p.turn.x_sh != p.turn.o_sh)) return KVE_EINVAL;
    p.turn.heads = hq;
  }
  if (n_tokens == 0) return KVE_OK;
  if (q) {   // the cache's device, or an address that the driver does not know
    const int device = place_of(q_out);
    if (device == kHostMemory || (device >= 0 && cache->device >= 0 && device != cache->device)) return KVE_EINVAL;
  }
  p.turn.r = rotary->table;
  p.turn.x = q;
  p.turn.out = q_out;
  p.turn.positions = positions;
  p.turn.n_tokens = n_tokens;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->bits == 4 ? kve::launch_cache4_append(p, st) : kve::launch_cache_append(p, st);
  return e == cudaSuccess ? KVE_OK : KVE_ECUDA;
}

kve_status kv_evict_cache_attend(const kve_cache* cache, int32_t layer, int32_t n_seq, int32_t q_tokens,
                                 const uint16_t* q, const int64_t* q_strides, const int32_t* table,
                                 const int32_t* lens, uint16_t* out, const int64_t* out_strides, float* lse,
                                 void* ws, void* stream) {
  if (!cache || !table || !lens || !ws || !aligned(ws, 256) || (n_seq != 0 && (!q || !out))) return KVE_EINVAL;
  const kve::CacheGeometry& c = cache->geo;
  if (layer < 0 || layer >= c.num_layers || n_seq < 0 || n_seq > c.max_seqs || q_tokens < 1 ||
      static_cast<int64_t>(q_tokens) * c.group > kve::kMaxRows)
    return KVE_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(table, 4) || !aligned(lens, 4) || !aligned(lse, 4))
    return KVE_EINVAL;
  kve::AttendParams p;
  std::memset(&p, 0, sizeof(p));
  if (!row_strides(q_strides, c.hq, &p.q_st, &p.q_sh) || !row_strides(out_strides, c.hq, &p.o_st, &p.o_sh))
    return KVE_EINVAL;
  const int64_t tokens = static_cast<int64_t>(n_seq) * q_tokens;
  if (!kve::rows_apart(tokens, p.o_st, c.hq, p.o_sh)) return KVE_EINVAL;
  if (!on_device(cache)) return KVE_EINVAL;
  if (n_seq == 0) return KVE_OK;
  if (cache->bits == 8 && !cache->maps) return KVE_ECUDA;
  p.c = c;
  p.wait_limit_ns = kWaitNs;
  p.n_seq = n_seq;
  p.q_tokens = q_tokens;
  p.alpha = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(kHeadDim)));
  p.group_inverse = 0xffffffffu / static_cast<uint32_t>(c.group) + 1u;
  p.q = q;
  p.out = out;
  p.lse = lse;
  p.table = table + static_cast<int64_t>(layer) * c.max_seqs * c.max_pages;
  p.lens = lens + static_cast<int64_t>(layer) * c.max_seqs;
  p.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + cache->ws.partial);
  p.arrive = word(ws, cache->ws.arrive);
  p.err = word(ws, cache->ws.err);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->bits == 4 ? kve::launch_cache4_attend(*cache, p, st) : kve::launch_cache_attend(*cache, p, st);
  return e == cudaSuccess ? KVE_OK : KVE_ECUDA;
}

kve_status kv_evict_cache_status(const kve_cache* cache, void* ws, void* stream) {
  if (!cache || !ws || !aligned(ws, 256) || !on_device(cache)) return KVE_EINVAL;
  // all on the caller's stream, so that its next call finds the words cleared
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const kve::CacheWsLayout& w = cache->ws;
  uint32_t err = 0;
  if (cudaMemcpyAsync(&err, word(ws, w.err), sizeof(err), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess)
    return KVE_ECUDA;
  if (err == 0) return KVE_OK;
  // the arrival counters too: a call that gave up may not have counted all of its parts; `refused` stays until
  // the next kv_evict_cache_pages call
  if (cudaMemsetAsync(ws, 0, w.refused, st) != cudaSuccess ||
      cudaMemsetAsync(word(ws, w.arrive), 0, w.clear_end - w.arrive, st) != cudaSuccess)
    return KVE_ECUDA;
  if (err & kve::kErrCheck) return KVE_ECUDA;
  return err & kve::kErrWait ? KVE_ETIMEOUT : KVE_EPAGES;
}

}  // extern "C"
