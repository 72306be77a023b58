// Rotary positions on the device: the turns of a position's pairs, and rows of bf16 turned by them.
#pragma once

#include "kve_internal.h"

namespace kve {

// {cos, sin} times the amplitude of the angle that pair j has at position pos. The angle is a fraction of a turn in 64-bit
// integers (exact for every position, where an fp32 product is off by 2^-24 of the whole angle); its upper 32 bits
// leave 1.5e-9 radians, and the approximate functions on [-pi, pi] an absolute 2^-20: 2^-11 of the bf16 rounding of what they
// turn.
__device__ __forceinline__ float2 turn_of(uint32_t hi, uint32_t lo, float amplitude, int pos) {
  const uint32_t p = static_cast<uint32_t>(pos);
  uint32_t u = p * hi + __umulhi(p, lo);
  if (pos < 0) u -= lo;   // (p is 2^32 too large)
  const float x = static_cast<float>(static_cast<int32_t>(u)) * 1.46291807926715968e-9f;   // pi 2^-31
  return make_float2(__cosf(x) * amplitude, __sinf(x) * amplitude);
}

// (a, b) turned: (a c - b s, b c + a s), each rounded once behind its second product.
__device__ __forceinline__ float2 turned(float a, float b, float2 cs) {
  return make_float2(fmaf(a, cs.x, -__fmul_rn(b, cs.y)), fmaf(b, cs.x, __fmul_rn(a, cs.y)));
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float bf16_low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// 16 elements of a row, 8 pairs: a and b are 8 elements and their partners, or 16 elements whose neighbours are partners.
__device__ __forceinline__ void turn_chunks(uint4& a, uint4& b, const float2 (&cs)[8], bool interleaved) {
  uint32_t* x = &a.x;
  uint32_t* y = &b.x;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = turned(bf16_low(x[i]), bf16_high(x[i]), cs[i]), v = turned(bf16_low(y[i]), bf16_high(y[i]), cs[4 + i]);
      x[i] = bf16_pair(u.x, u.y);
      y[i] = bf16_pair(v.x, v.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = turned(bf16_low(x[i]), bf16_low(y[i]), cs[2 * i]);
      const float2 v = turned(bf16_high(x[i]), bf16_high(y[i]), cs[2 * i + 1]);
      x[i] = bf16_pair(u.x, v.x);
      y[i] = bf16_pair(u.y, v.y);
    }
  }
}

// Which 8-element chunks lane l of the 8 that share a row has, and whether they are turned.
struct RowChunks {
  int a, b;
  bool turns;
};
__device__ __forceinline__ RowChunks row_chunks(const RotaryTable& r, int l) {
  const int half = r.pairs >> 3;   // lanes that turn: 8 pairs each
  if (l >= half || r.interleaved) return {2 * l, 2 * l + 1, l < half};
  return {l, l + half, true};
}

// The turns of `tokens` tokens from `token0` on into shared memory, [tokens][kMaxPairs]; every thread comes here and meets
// the others behind it.
__device__ __forceinline__ void turns_to_shared(float2* to, const RotaryTable& r, const int32_t* positions, int64_t token0,
                                                int tokens, bool transpose) {
  for (int i = threadIdx.x; i < tokens * kMaxPairs; i += blockDim.x) {
    const int j = i % kMaxPairs;
    if (j >= r.pairs) continue;
    float2 cs = turn_of(r.hi[j], r.lo[j], r.amplitude, __ldg(positions + token0 + i / kMaxPairs));
    if (transpose) cs.y = -cs.y;
    to[i] = cs;
  }
  __syncthreads();
}

__device__ __forceinline__ void lane_turns(float2 (&cs)[8], const float2* token_turns, int l) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(token_turns + 8 * l)[i];
    cs[2 * i] = make_float2(v.x, v.y);
    cs[2 * i + 1] = make_float2(v.z, v.w);
  }
}

// One CTA's tile of rows: 8 lanes a row, 32 bytes a lane; a lane keeps the turns of its token and goes through heads, four
// rows in flight. turns: kTileTokens * kMaxPairs of shared memory, 16-byte aligned.
constexpr int kTurnTokens = 8;
template <int kThreads>
__device__ __forceinline__ void rotate_tile(const RotateParams& P, int64_t tile, float2* turns) {
  constexpr int kGroups = kThreads / 8, kInFlight = 4;
  const int head_tiles = (P.heads + P.tile_heads - 1) / P.tile_heads;
  const int64_t token0 = tile / head_tiles * P.tile_tokens;
  const int head0 = static_cast<int>(tile % head_tiles) * P.tile_heads;
  const int tokens = static_cast<int>(P.n_tokens - token0 < P.tile_tokens ? P.n_tokens - token0 : P.tile_tokens);
  turns_to_shared(turns, P.r, P.positions, token0, tokens, P.transpose);
  const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
  const int tok = group % P.tile_tokens, step = kGroups / P.tile_tokens;
  if (tok >= tokens) return;
  const RowChunks c = row_chunks(P.r, l);
  if (!c.turns && P.out == P.x) return;
  float2 cs[8];
  if (c.turns) lane_turns(cs, turns + tok * kMaxPairs, l);
  const uint16_t* x = P.x + (token0 + tok) * P.x_st;
  uint16_t* out = P.out + (token0 + tok) * P.o_st;
  const int end = min(head0 + P.tile_heads, P.heads);
  for (int h = head0 + group / P.tile_tokens; h < end; h += kInFlight * step) {
    uint4 a[kInFlight], b[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (h + i * step < end) {
        const uint4* from = reinterpret_cast<const uint4*>(x + (h + i * step) * P.x_sh);
        a[i] = from[c.a];
        b[i] = from[c.b];
      }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (h + i * step < end) {
        if (c.turns) turn_chunks(a[i], b[i], cs, P.r.interleaved);
        uint4* to = reinterpret_cast<uint4*>(out + (h + i * step) * P.o_sh);
        to[c.a] = a[i];
        to[c.b] = b[i];
      }
  }
}

// Tiles of a call for CTAs of kThreads threads, and their number: 8 tokens (or fewer, a power of two), whose turns are
// computed once, by as many heads as give a thread four rows, or one row where that leaves SMs without work.
template <int kThreads>
inline int64_t cut_rotate(RotateParams& p) {
  p.tile_tokens = kTurnTokens;
  while (p.tile_tokens > 1 && p.tile_tokens / 2 >= p.n_tokens) p.tile_tokens /= 2;
  const int step = kThreads / 8 / p.tile_tokens;
  const auto tiles = [&](int heads) {
    return (p.n_tokens + p.tile_tokens - 1) / p.tile_tokens * ((p.heads + heads - 1) / heads);
  };
  p.tile_heads = 4 * step;
  if (tiles(p.tile_heads) < 304) p.tile_heads = step;
  return tiles(p.tile_heads);
}

}  // namespace kve
