// Rows of the paged 4-bit cache: the kept and the window rows of an eviction, and new tokens by slot, with or without the
// rotation of their keys (and queries) on the way.
//
// A row x (128 elements, finite) becomes 128 codes and two bf16 numbers:
//   z = min x,   s = RN_bf16((max x - min x) / 15),   c = RN((x - z) / s) in 0 .. 15
// (s = 0, c = 0 where s would be below 2^-120; a row with an infinity or a NaN is a row of NaN: s = z = NaN, c = 0). No
// row shares anything with another, so a page can be written row by row in any order, and a token that joins a page
// touches no older one. s is rounded to 8 bits because c is chosen with the rounded s: it costs a 2^-9 of the range at
// the far end, a 30th of a code's half step; z is an element and so exact.
//
// Bound by HBM: 256 bytes read and 68 written a row. Eight lanes have a row, 16 elements (32 bytes) each; the minimum
// and maximum are packed bf16 operations and three shuffles, the division one reciprocal a row. 23,815 tokens of 8 heads (123 MB)
// are stored in 24.1 us (18.5 at the copy's rate); 256 tokens in 1.8, which is the launch and two loads in a row (slots, rows).
#include "kve_ptx.cuh"
#include "kve_rotary.cuh"

namespace kve {
namespace {

constexpr int kRowThreads4 = 256;
constexpr int kGroups4 = kRowThreads4 / 8;
constexpr int kRowCodes = kHeadDim / 2;   // bytes
constexpr int kStoreTokens = kGroups4;    // most tokens of a tile

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

// Writes row `row` (negative: nothing) that 8 lanes hold in the chunks ca and cb: its codes, and in lane l = 0 its s and z. Whole
// warps call it: shuffles under a mask of some lanes only cost more than the rows that are not there.
__device__ __forceinline__ void write_row4(const uint4& a, const uint4& b, int ca, int cb, uint8_t* codes, uint32_t* param,
                                           int row, int l) {
  const uint32_t lo = min2(min2(min2(a.x, a.y), min2(a.z, a.w)), min2(min2(b.x, b.y), min2(b.z, b.w))) ^ 0x80008000u;
  const uint32_t hi = max2(max2(max2(a.x, a.y), max2(a.z, a.w)), max2(max2(b.x, b.y), max2(b.z, b.w)));
  // the largest in the low half, minus the least in the high half
  uint32_t ends = max2(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632));
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) ends = max2(ends, __shfl_xor_sync(0xffffffffu, ends, o));
  const bool finite = (ends & 0x7f80u) != 0x7f80u && (ends & 0x7f800000u) != 0x7f800000u;
  // in units of 16, so that no difference overflows
  const float less = bf16_high(ends), z16 = less * -0.0625f;
  const float spread16 = fmaf(bf16_low(ends), 0.0625f, -z16);
  uint32_t s = bf16_pair(spread16 * 1.0666666667f, 0.f - less);   // 16 / 15
  if (bf16_low(s) < 7.52316384526264e-37f) s &= 0xffff0000u;      // 2^-120
  const float unit = bf16_low(s) * 0.0625f;
  const bool spread = finite && unit > 0.f;
  const float inverse = rcp(unit), rest = fmaf(-unit, inverse, 1.f) * inverse;
  const uint32_t first = spread ? codes_of(a, z16, inverse, rest) : 0u, second = spread ? codes_of(b, z16, inverse, rest) : 0u;
  if (row < 0) return;
  uint32_t* const to = reinterpret_cast<uint32_t*>(codes + static_cast<int64_t>(row) * kRowCodes);
  to[ca] = first;
  to[cb] = second;
  if (l == 0) param[row] = finite ? s : 0x7fc07fc0u;
}

// New tokens by slot. A tile is up to kStoreTokens tokens by some heads of keys or of values (the two alternate). With kTurn
// the last tiles turn the queries, and keys are turned (and rounded to bf16) before they are coded.
template <bool kTurn>
__global__ void __launch_bounds__(kRowThreads4) cache4_store_kernel(const __grid_constant__ CacheAppendParams A, int tile_tokens,
                                                                    int tile_heads, uint32_t row_tiles) {
  wait_previous_kernel();
  __shared__ __align__(16) float2 turns[kTurn ? kStoreTokens * kMaxPairs : 1];
  const CacheStoreParams& P = A.s;
  uint32_t tile = blockIdx.x;
  if constexpr (kTurn) {
    if (tile >= row_tiles) {
      rotate_tile<kRowThreads4>(A.turn, tile - row_tiles, turns);
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
  const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
  const int tok = group & (tile_tokens - 1), step = kGroups4 / tile_tokens;
  const int slot = tok < tokens ? __ldg(P.slots + token0 + tok) : -1;
  RowChunks kc = {l, l + 8, false, false};
  if constexpr (kTurn) {
    if (key) kc = row_chunks(A.turn.r, l);
  }
  const int end = tok < tokens ? min(head0 + tile_heads, H) : 0;
  constexpr int kInFlight = 4;
  const uint16_t* const base = key ? P.k + (token0 + tok) * P.k_st : P.v + (token0 + tok) * P.v_st;
  const int64_t across = key ? P.k_sh : P.v_sh;
  uint8_t* const codes = key ? P.c.k : P.c.v;
  uint32_t* const param = key ? P.c.k_param : P.c.v_param;
  uint4 a[kInFlight], b[kInFlight];
  const auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (h + i * step < end) {
        const uint4* from = reinterpret_cast<const uint4*>(base + (h + i * step) * across);
        a[i] = from[kc.a];
        b[i] = from[kc.b];
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
        if (key) turn_chunks(a[i], b[i], cs, kc, A.turn.r.interleaved);
      }
      write_row4(a[i], b[i], kc.a, kc.b, codes, param, there ? row0 + ((h + i * step) << P.c.page_shift) : -1, l);
    }
    h += kInFlight * step;
    load(h);
  }
  allow_next_kernel();
}

// Step 4 into the cache: 8 lanes a row, of keys and of values, kGatherTurns times with the next row's place looked up ahead.
// Reads whole rows at random places and writes a row's 64 bytes and its numbers: 16 requests of 509 kept rows and 8 layers, 327 MB,
// take 62.4 us of 48.9 at the copy's rate, 64 requests' smallest (32 layers of 72 rows) 4.9 of 2.4. Tiles of 32 rows (one turn)
// take 83.7 and 4.6, of 256 rows 62.2 and 5.0; two rows of a lane in flight, with 3 CTAs an SM for their registers, 82.0 and 4.95.
constexpr int kGatherTurns = 4;
constexpr int kGatherTile = kGroups4 * kGatherTurns;   // rows of a unit that a CTA has
__global__ void __launch_bounds__(kRowThreads4, 5) cache4_gather_kernel(const __grid_constant__ CacheGatherParams P,
                                                                         uint32_t unit_tiles) {
  wait_previous_kernel();   // the indices come from the selection launched before
  const uint32_t unit = blockIdx.x / unit_tiles;
  const int tile = static_cast<int>(blockIdx.x - unit * unit_tiles);
  const UnitInfo u = unit_info(P.g.g, unit);
  const int W = P.g.g.window, Lc = u.L - W;
  const int m = min(P.g.layer_budget[u.layer], Lc), n = m + W;
  const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
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
  for (int row = first; row - (group & 3) < end; row += kGroups4) {   // (the warp's first row)
    uint4 k[2] = {}, v[2] = {};
    const bool there = row < end;
    const bool outside = row < m && static_cast<uint32_t>(src) >= static_cast<uint32_t>(Lc);   // never read outside the unit
    const bool good = static_cast<uint32_t>(page) < static_cast<uint32_t>(P.c.num_pages);
    if (there && (outside || !good) && l == 0) atomicOr(P.err, kErrCheck);
    const int at = there && good ? (page * P.c.heads << shift) + head + (row & (P.c.page - 1)) : -1;
    if (there && !outside) {   // (else a row of zeros)
      const uint4* ks = reinterpret_cast<const uint4*>(P.g.k + u.k_off + src * P.g.g.k_st) + l;
      const uint4* vs = reinterpret_cast<const uint4*>(P.g.v + u.v_off + src * P.g.g.v_st) + l;
      k[0] = __ldg(ks);
      k[1] = __ldg(ks + 8);
      v[0] = __ldg(vs);
      v[1] = __ldg(vs + 8);
    }
    look_up(row + kGroups4);
    write_row4(k[0], k[1], l, l + 8, P.c.k, P.c.k_param, at, l);
    write_row4(v[0], v[1], l, l + 8, P.c.v, P.c.v_param, at, l);
  }
  allow_next_kernel();
}

template <bool kTurn>
cudaError_t store4(CacheAppendParams p, cudaStream_t stream) {
  const int64_t turn_tiles = kTurn && p.turn.heads > 0 ? cut_rotate<kRowThreads4>(p.turn) : 0;
  RotateParams cut;
  cut.n_tokens = p.s.n_tokens;
  cut.heads = p.s.c.heads;
  int64_t tiles = cut_rotate<kRowThreads4>(cut);
  // A group a token and all its heads one after the other, where that still gives every SM a tile of keys and one of values: 24k
  // tokens 24.1 us. (With it and without: 2500 tokens of 8 heads 5.6 and 4.4 us, 5000 7.35 and 7.3, 10000 13.6 and 15.2.)
  if (cut.n_tokens >= 152 * kStoreTokens) {
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
  return launch_after_previous(cache4_gather_kernel, dim3(static_cast<unsigned>(p.g.g.n_units * tiles)), dim3(kRowThreads4), 0,
                               stream, p, static_cast<uint32_t>(tiles));
}

}  // namespace kve
