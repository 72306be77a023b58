// Rows of the paged 4-bit cache: the kept and the window rows of an eviction, and new tokens by slot, with or without the
// rotation of their keys (and queries) on the way.
//
// A row x (128 elements, finite) becomes 128 codes and two bf16 numbers:
//   z = min x,   s = RN_bf16((max x - min x) / 15),   c = RN((x - z) / s) in 0 .. 15
// with differences and the quotient in fp32, in units of 16 so that none overflows, and the fifteenth as a product with fl(16 / 15)
// (5.6e-8 above it: of the ends of 400,000 normal rows it rounds none to another s than a division, of 4M pairs of normal ends 2228)
// (s = 0, c = 0 where s would be below 2^-120; a row with an infinity or a NaN is a row of NaN: s = z = NaN, c = 0). No
// row shares anything with another, so a page can be written row by row in any order, and a token that joins a page
// touches no older one. s is rounded to 8 bits because c is chosen with the rounded s: it costs a 2^-9 of the range at
// the far end, a 30th of a code's half step; z is an element and so exact.
//
// Bound by HBM: 256 bytes read and 68 written a row. Four lanes have a row, 64 bytes each as two pieces of 32 (with turns eight, as
// the pairs lie); the minimum and maximum are packed bf16 operations and two shuffles, the division one reciprocal a row. What a row
// costs beside its elements is half of the instructions, so few lanes a row and many rows an SM.
#include "kve_ptx.cuh"
#include "kve_rotary.cuh"

namespace kve {
namespace {

constexpr int kRowThreads4 = 256;
constexpr int kRowCodes = kHeadDim / 2;   // bytes
constexpr int kStoreTokens = 32;          // most tokens of a tile

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The codes of 8 elements, the first in the lowest four bits: (x - z) / s in 0 .. 15.06 (s is off by at most 2^-8) to the nearest,
// ties to the even one. With inverse + rest = 1 / unit to 2^-44 of itself, q is the quotient rounded to fp32 as a division
// rounds it: a quotient of a float by one of 8 bits is no nearer than 2^-33 of itself to the middle between two floats
// without being a float.
__device__ __forceinline__ uint32_t codes_of(const uint4& x, float z16, float inverse, float rest) {
  const uint32_t* w = &x.x;
  const float2 scale = make_float2(0.0625f, 0.0625f), z = make_float2(-z16, -z16);
  const float2 hi = make_float2(inverse, inverse), lo = make_float2(rest, rest);
  constexpr float kWhole = 12582912.f;   // 1.5 * 2^23: a sum with it has its integer in the low bits, 0x4b400000 above
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 d = ffma2(make_float2(bf16_low(w[i]), bf16_high(w[i])), scale, z);
    const float2 t = fadd2(ffma2(d, hi, fmul2(d, lo)), make_float2(kWhole, kWhole));
    u[2 * i] = __float_as_uint(t.x);
    u[2 * i + 1] = __float_as_uint(t.y);
  }
  // sum of u_i 16^i, without 0x4b400000 * 0x11111111 (modulo 2^32)
  uint32_t out = u[7];
#pragma unroll
  for (int i = 6; i >= 0; --i) out = out * 16u + u[i];
  return out - 0x4b400000u * 0x11111111u;
}

// The codes of row `row` (negative: nothing) that 16 / N lanes hold, N chunks of 8 elements each, and in lane l = 0 its s and z.
// Whole warps come here: shuffles under a mask of some lanes only cost more than the rows that are not there.
template <int N>
__device__ __forceinline__ void row_codes4(const uint4 (&x)[N], uint32_t (&c)[N], uint32_t* param, int row, int l) {
  uint32_t lo = 0, hi = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t a = min2(min2(x[i].x, x[i].y), min2(x[i].z, x[i].w)), b = max2(max2(x[i].x, x[i].y), max2(x[i].z, x[i].w));
    lo = i ? min2(lo, a) : a;
    hi = i ? max2(hi, b) : b;
  }
  lo ^= 0x80008000u;
  // the largest in the low half, minus the least in the high half
  uint32_t ends = max2(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632));
#pragma unroll
  for (int o = 8 / N; o > 0; o >>= 1) ends = max2(ends, __shfl_xor_sync(0xffffffffu, ends, o));
  const bool finite = (ends & 0x7f80u) != 0x7f80u && (ends & 0x7f800000u) != 0x7f800000u;
  // in units of 16, so that no difference overflows
  const float less = bf16_high(ends), z16 = less * -0.0625f;
  const float spread16 = fmaf(bf16_low(ends), 0.0625f, -z16);
  uint32_t s = bf16_pair(spread16 * 1.0666666667f, 0.f - less);   // 16 / 15
  if (bf16_low(s) < 7.52316384526264e-37f) s &= 0xffff0000u;      // 2^-120
  const float unit = bf16_low(s) * 0.0625f;
  const bool spread = finite && unit > 0.f;
  const float inverse = rcp(unit), rest = fmaf(-unit, inverse, 1.f) * inverse;
#pragma unroll
  for (int i = 0; i < N; ++i) c[i] = spread ? codes_of(x[i], z16, inverse, rest) : 0u;
  if (row >= 0 && l == 0) param[row] = finite ? s : 0x7fc07fc0u;
}

__device__ __forceinline__ void write_codes4(const uint32_t (&c)[2], uint8_t* codes, int row, int, const RowChunks& at) {
  uint32_t* const to = reinterpret_cast<uint32_t*>(codes + static_cast<int64_t>(row) * kRowCodes);
  to[at.a] = c[0];
  to[at.b] = c[1];
}
__device__ __forceinline__ void write_codes4(const uint32_t (&c)[4], uint8_t* codes, int row, int l, const RowChunks& = {}) {
  uint2* const to = reinterpret_cast<uint2*>(codes + static_cast<int64_t>(row) * kRowCodes);
  to[l] = make_uint2(c[0], c[1]);
  to[l + 4] = make_uint2(c[2], c[3]);
}

// New tokens by slot. A tile is up to kStoreTokens tokens by some heads of keys or of values (the two alternate). With kTurn
// the last tiles turn the queries, and keys are turned (and rounded to bf16) before they are coded.
//
// Without turns a lane has one row in flight and an SM 56 warps: 23,815 tokens of 8 heads (123 MB) 22.9 us of 18.5, 10,000 10.8,
// 1000 2.3; two rows and 40 warps took 26.4, 12.8 and 2.4, with 8 lanes a row 23.5, 13.1 and 2.9. Its 32 registers spill 44 bytes: with 48
// warps and 12 bytes 23.9, 11.5 and 2.25, with 40 and none 25.0, 12.1 and 2.2. With turns four rows and 32 warps: those tokens with 32
// query heads (514 MB) 84.2 us of 76.9, 1000 x 8 tokens 31.2, 256 3.7, 16 2.7, whatever the page. 64 registers spill 96 bytes; 24 warps
// and no spills take 84.2, 30.6, 3.4 and 2.45; two rows and 40 warps spill more (158).
template <bool kTurn>
__global__ void __launch_bounds__(kRowThreads4, kTurn ? 4 : 7) cache4_store_kernel(const __grid_constant__ CacheAppendParams A, int tile_tokens,
                                                                    int tile_heads, uint32_t row_tiles) {
  wait_previous_kernel();
  __shared__ __align__(16) float2 turns[kTurn ? kStoreTokens * kMaxPairs : 1];
  const CacheStoreParams& P = A.s;
  uint32_t tile = blockIdx.x;
  if constexpr (kTurn) {
    if (tile >= row_tiles) {
      rotate_tile<kRowThreads4, 4>(A.turn, tile - row_tiles, turns);
      allow_next_kernel();
      return;
    }
  }
  const int H = P.c.heads;
  const bool key = (tile & 1) == 0;
  tile >>= 1;
  const uint32_t head_tiles = static_cast<uint32_t>((H + tile_heads - 1) / tile_heads);
  const int64_t token0 = static_cast<int64_t>(tile / head_tiles) * tile_tokens;
  const int head0 = static_cast<int>(tile % head_tiles) * tile_heads;
  const int tokens = static_cast<int>(P.n_tokens - token0 < tile_tokens ? P.n_tokens - token0 : tile_tokens);
  constexpr int N = kTurn ? 2 : 4, kLanes = 16 / N;   // chunks of 8 elements a lane, lanes a row
  const int l = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int tok = group & (tile_tokens - 1), step = kRowThreads4 / kLanes / tile_tokens;
  const int slot = tok < tokens ? __ldg(P.slots + token0 + tok) : -1;
  RowChunks kc = {l, l + 8, false, false};   // (kTurn; else the chunks 2 l, 2 l + 1 and those 8 further on)
  if constexpr (kTurn) {
    if (key) kc = row_chunks(A.turn.r, l);
  }
  const auto chunk = [&](int c) { return kTurn ? (c ? kc.b : kc.a) : 2 * l + (c & 1) + 8 * (c >> 1); };
  const int end = tok < tokens ? min(head0 + tile_heads, H) : 0;
  constexpr int kInFlight = kTurn ? 4 : 1;   // rows of a lane
  const uint16_t* const base = key ? P.k + (token0 + tok) * P.k_st : P.v + (token0 + tok) * P.v_st;
  const int64_t across = key ? P.k_sh : P.v_sh;
  uint8_t* const codes = key ? P.c.k : P.c.v;
  uint32_t* const param = key ? P.c.k_param : P.c.v_param;
  uint4 x[kInFlight][N];
  const auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (h + i * step < end) {
        const uint4* from = reinterpret_cast<const uint4*>(base + (h + i * step) * across);
#pragma unroll
        for (int c = 0; c < N; ++c) x[i][c] = from[chunk(c)];
      }
  };
  int h = head0 + group / tile_tokens;
  load(h);
  float2 cs[8];
  if constexpr (kTurn) {
    if (key) {
      turns_to_shared<kRowThreads4>(turns, A.turn.r, A.turn.positions, token0, tokens, false);
      if (tok < tokens && kc.turns_a) lane_turns(cs, turns + tok * kMaxPairs, A.turn.r, kc);
    }
  }
  const int limit = P.c.num_pages << P.c.page_shift;   // (below 2^31)
  if (slot >= limit && l == 0 && group / tile_tokens == 0) atomicOr(P.err, kErrCheck);
  const bool kept = slot >= 0 && slot < limit;
  // rows of the pool are below 2^31
  const int row0 = ((slot >> P.c.page_shift) * H << P.c.page_shift) + (slot & (P.c.page - 1));
  while (__any_sync(0xffffffffu, kept && h < end)) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const bool there = kept && h + i * step < end;
      if (!__any_sync(0xffffffffu, there)) break;
      if constexpr (kTurn) {
        if (key) turn_chunks(x[i][0], x[i][1], cs, kc, A.turn.r.interleaved);
      }
      const int row = there ? row0 + ((h + i * step) << P.c.page_shift) : -1;
      uint32_t c[N];
      row_codes4<N>(x[i], c, param, row, l);
      if (there) write_codes4(c, codes, row, l, kc);
    }
    h += kInFlight * step;
    load(h);
  }
  allow_next_kernel();
}

// Step 4 into the cache: a CTA has keys or values of a unit, 4 lanes a row, kGatherTurns rows one after the other with the next
// one's place looked up ahead. Whole rows at random places: 16 requests of 509 + 8 rows in 8 layers (327 MB) take 54.1 us of 48.9 at
// a copy's rate, 32 layers of one request's 96 rows 4.5 of 2.4 (12 bytes of spills; without, at 6 CTAs an SM, 56.1 and 4.5). With 8 lanes a row and keys and values in one CTA 61.5 and 4.9; with
// 2 rows a CTA 66 and 4.4, with 8 57.1 and 4.6; with 5 CTAs an SM 60.5.
constexpr int kGatherTurns = 4, kGatherGroups = kRowThreads4 / 4;
constexpr int kGatherTile = kGatherGroups * kGatherTurns;   // rows of a unit that a CTA has
__global__ void __launch_bounds__(kRowThreads4, 7) cache4_gather_kernel(const __grid_constant__ CacheGatherParams P,
                                                                         uint32_t unit_tiles) {
  wait_previous_kernel();   // the indices come from the selection launched before
  const bool key = (blockIdx.x & 1) == 0;
  const uint32_t unit = (blockIdx.x >> 1) / unit_tiles;
  const int tile = static_cast<int>((blockIdx.x >> 1) - unit * unit_tiles);
  const UnitInfo u = unit_info(P.g.g, unit);
  const int W = P.g.g.window, Lc = u.L - W;
  const int m = min(P.g.layer_budget[u.layer], Lc), n = m + W;
  const int l = threadIdx.x & 3, group = threadIdx.x >> 2;
  const int first = tile * kGatherTile + group, end = min(n, (tile + 1) * kGatherTile);
  const bool refused = __ldg(P.refused) != 0;   // the table's pages may be other sequences' by now
  const int32_t* const table = P.table + (static_cast<int64_t>(u.layer) * P.c.max_seqs + P.first_seq + u.r) * P.c.max_pages;
  const int32_t* const indices = P.g.indices + static_cast<int64_t>(unit) * P.g.budget;
  const int shift = P.c.page_shift, head = u.h << shift;
  if (refused) return;
  // where the row comes from and its page, a turn ahead
  int src = 0, page = 0;
  const auto look_up = [&](int row) {
    if (row >= end) return;
    page = __ldg(table + (row >> shift));
    src = row < m ? __ldg(indices + row) : Lc + (row - m);
  };
  look_up(first);
  const uint16_t* const from = key ? P.g.k + u.k_off : P.g.v + u.v_off;
  const int64_t st = key ? P.g.g.k_st : P.g.g.v_st;
  uint8_t* const codes = key ? P.c.k : P.c.v;
  uint32_t* const param = key ? P.c.k_param : P.c.v_param;
  for (int row = first; row - (group & 7) < end; row += kGatherGroups) {   // (the warp's first row)
    uint4 x[4] = {};
    const bool there = row < end;
    const bool outside = row < m && static_cast<uint32_t>(src) >= static_cast<uint32_t>(Lc);   // never read outside the unit
    const bool good = static_cast<uint32_t>(page) < static_cast<uint32_t>(P.c.num_pages);
    if (there && (outside || !good) && l == 0) atomicOr(P.err, kErrCheck);
    const int at = there && good ? (page * P.c.heads << shift) + head + (row & (P.c.page - 1)) : -1;
    if (there && !outside) {   // (else a row of zeros)
      const uint4* const xs = reinterpret_cast<const uint4*>(from + src * st) + 2 * l;
      x[0] = __ldg(xs);
      x[1] = __ldg(xs + 1);
      x[2] = __ldg(xs + 8);
      x[3] = __ldg(xs + 9);
    }
    look_up(row + kGatherGroups);
    uint32_t c[4];
    row_codes4<4>(x, c, param, at, l);
    if (at >= 0) write_codes4(c, codes, at, l);
  }
  allow_next_kernel();
}

template <bool kTurn>
cudaError_t store4(CacheAppendParams p, cudaStream_t stream) {
  const int64_t turn_tiles = kTurn && p.turn.heads > 0 ? cut_rotate<kRowThreads4>(p.turn) : 0;
  RotateParams cut;
  cut.n_tokens = p.s.n_tokens;
  cut.heads = p.s.c.heads;
  constexpr int kWide = kTurn ? kRowThreads4 : 2 * kRowThreads4;   // (8 lanes a row there)
  int64_t tiles = cut_rotate<kWide>(cut);
  // With turns, a group a token and all its heads one after the other, where that still gives every SM a tile of keys and one of
  // values: 6000 tokens 26.2 us for 31.3, 24k 95 for 117 at the time (24.7 and 84.2 now).
  if (kTurn && cut.n_tokens >= 152 * kStoreTokens) {
    cut.tile_tokens = kStoreTokens;
    cut.tile_heads = cut.heads;
    tiles = (cut.n_tokens + kStoreTokens - 1) / kStoreTokens;
  }
  tiles *= 2;   // of keys, and as many of values
  return launch_after_previous(cache4_store_kernel<kTurn>, dim3(static_cast<unsigned>(turn_tiles + tiles)), dim3(kRowThreads4), 0,
                               stream, p, cut.tile_tokens, cut.tile_heads, static_cast<uint32_t>(tiles));
}

}  // namespace

cudaError_t launch_cache4_store(const CacheStoreParams& s, cudaStream_t stream) {
  CacheAppendParams p = {};
  p.s = s;
  return store4<false>(p, stream);
}

cudaError_t launch_cache4_append(const CacheAppendParams& p, cudaStream_t stream) { return store4<true>(p, stream); }

cudaError_t launch_cache4_gather(const CacheGatherParams& p, cudaStream_t stream) {
  const int64_t rows = static_cast<int64_t>(p.unit_pages) << p.c.page_shift;
  const int64_t tiles = (rows + kGatherTile - 1) / kGatherTile;
  return launch_after_previous(cache4_gather_kernel, dim3(static_cast<unsigned>(p.g.g.n_units * tiles * 2)), dim3(kRowThreads4), 0,
                               stream, p, static_cast<uint32_t>(tiles));
}

}  // namespace kve
