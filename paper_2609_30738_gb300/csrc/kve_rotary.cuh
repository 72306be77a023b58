// Rotary positions on the device: the turns of a position's pairs, and rows of bf16 turned by them.
#pragma once

#include "kve_internal.h"
#include "kve_ptx.cuh"

namespace kve {

// turns[j] of a kernel parameter. The lanes ask for different j, which a read of the constant bank would serve one after the
// other: read as ordinary memory.
__device__ __forceinline__ uint2 turn_at(const RotaryTable& r, int j) {
  uint2 v;
  asm("ld.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(r.turns + j));
  return v;
}

// {cos, sin} times the amplitude of the angle that a pair has at position pos. The angle is a fraction of a turn in 64-bit
// integers (exact for every position, where an fp32 product is off by 2^-24 of the whole angle); its upper 32 bits are cut into
// the nearest quarter turn, which says which of the two is which and their signs, and a rest x of at most pi / 4, whose sine over x and
// cosine are their Taylor polynomials up to x^10 in packed fp32 (2^-32 off at pi / 4): 2^-23 with the roundings, half of it those of x.
// (Half turns, with polynomials up to x^14, were off by 2^-22.1: of 2M turned elements 95 went to another bf16 number than the exact result does,
// now 68, and 61 where cos and sin are rounded from 64 bits and each product by itself.)
__device__ __forceinline__ float2 turn_of(uint2 turn, float amplitude, int pos) {
  const uint32_t u = static_cast<uint32_t>(pos) * turn.y + static_cast<uint32_t>(__mulhi(pos, static_cast<int32_t>(turn.x)));
  const float x = static_cast<float>(static_cast<int32_t>(u << 2)) * 3.65729519816788900e-10f;   // pi 2^-33
  const float y = x * x;
  const float2 yy = make_float2(y, y);
  float2 p = ffma2(yy, make_float2(-2.50521084e-8f, -2.75573192e-7f), make_float2(2.75573192e-6f, 2.48015873e-5f));
  p = ffma2(yy, p, make_float2(-1.98412698e-4f, -1.38888889e-3f));
  p = ffma2(yy, p, make_float2(8.33333333e-3f, 4.16666667e-2f));
  p = ffma2(yy, p, make_float2(-1.66666667e-1f, -0.5f));
  p = ffma2(yy, p, make_float2(1.f, 1.f));
  const float s = p.x * x;
  // quarters 1 and 3 change places; the cosine is negative in 1 and 2, the sine in 2 and 3
  const uint32_t w = u + 0x20000000u;
  const bool odd = (w & 0x40000000u) != 0;
  const float a = __uint_as_float(__float_as_uint(amplitude) ^ ((w + 0x40000000u) & 0x80000000u));
  const float b = __uint_as_float(__float_as_uint(amplitude) ^ (w & 0x80000000u));
  return make_float2((odd ? s : p.y) * a, (odd ? p.y : s) * b);
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

// Four pairs, (a_i, b_i) by halves of x and y, or neighbours in x and y, with the turns cs[0 .. 3].
__device__ __forceinline__ void turn_halves(uint32_t (&x)[2], uint32_t (&y)[2], const float2* cs) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // two pairs at once, as `turned`
    const float2 a = make_float2(bf16_low(x[i]), bf16_high(x[i])), b = make_float2(bf16_low(y[i]), bf16_high(y[i]));
    const float2 c = make_float2(cs[2 * i].x, cs[2 * i + 1].x), s = make_float2(cs[2 * i].y, cs[2 * i + 1].y);
    const float2 u = ffma2(a, c, fmul2(b, make_float2(-s.x, -s.y))), v = ffma2(b, c, fmul2(a, s));
    x[i] = bf16_pair(u.x, u.y);
    y[i] = bf16_pair(v.x, v.y);
  }
}
__device__ __forceinline__ void turn_neighbours(uint4& x, const float2* cs) {
  uint32_t* w = &x.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 u = turned(bf16_low(w[i]), bf16_high(w[i]), cs[i]);
    w[i] = bf16_pair(u.x, u.y);
  }
}

// Which 8-element chunks lane l of the 8 that share a row has, and which of them are turned. Chunks of the 8 lanes stand side by
// side (128 bytes of the row at once), but for parts of a row that turn by halves.
struct RowChunks {
  int a, b;
  bool turns_a, turns_b;
};
__device__ __forceinline__ RowChunks row_chunks(const RotaryTable& r, int l) {
  const int half = r.pairs >> 3;   // chunks of first elements
  if (r.interleaved) return {l, l + 8, l < 2 * half, l + 8 < 2 * half};
  return l < half ? RowChunks{l, l + half, true, true} : RowChunks{l + half, l + 8, false, false};
}

// The turns of those chunks: of the pairs of both, or of each one's.
__device__ __forceinline__ void lane_turns(float2 (&cs)[8], const float2* token_turns, const RotaryTable& r, const RowChunks& c) {
  const int j0 = r.interleaved ? 4 * c.a : 8 * c.a, j1 = r.interleaved ? 4 * c.b : j0 + 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(token_turns + (i < 2 ? j0 : j1))[i & 1];
    cs[2 * i] = make_float2(v.x, v.y);
    cs[2 * i + 1] = make_float2(v.z, v.w);
  }
}

__device__ __forceinline__ void turn_chunks(uint4& a, uint4& b, const float2 (&cs)[8], const RowChunks& c, bool interleaved) {
  if (interleaved) {
    if (c.turns_a) turn_neighbours(a, cs);
    if (c.turns_b) turn_neighbours(b, cs + 4);
  } else if (c.turns_a) {
    uint32_t x0[2] = {a.x, a.y}, x1[2] = {a.z, a.w}, y0[2] = {b.x, b.y}, y1[2] = {b.z, b.w};
    turn_halves(x0, y0, cs);
    turn_halves(x1, y1, cs + 4);
    a = make_uint4(x0[0], x0[1], x1[0], x1[1]);
    b = make_uint4(y0[0], y0[1], y1[0], y1[1]);
  }
}

// The turns of `tokens` tokens from `token0` on into shared memory, [tokens][kMaxPairs]; every thread comes here and meets
// the others behind it.
template <int kThreads>
__device__ __forceinline__ void turns_to_shared(float2* to, const RotaryTable& r, const int32_t* positions, int64_t token0,
                                                int tokens, bool transpose) {
  static_assert(kThreads % kMaxPairs == 0, "a thread has one pair");
  const int j = threadIdx.x % kMaxPairs;
  if (j < r.pairs) {
    const uint2 turn = turn_at(r, j);
    for (int i = threadIdx.x / kMaxPairs; i < tokens; i += kThreads / kMaxPairs) {
      float2 cs = turn_of(turn, r.amplitude, __ldg(positions + token0 + i));
      if (transpose) cs.y = -cs.y;
      to[i * kMaxPairs + j] = cs;
    }
  }
  __syncthreads();
}

// One CTA's tile of rows: 8 lanes a row, 32 bytes a lane; a lane keeps the turns of its token and goes through heads,
// kInFlight rows in flight. turns: kTileTokens * kMaxPairs of shared memory, 16-byte aligned.
constexpr int kTurnTokens = 8;
template <int kThreads, int kInFlight>
__device__ __forceinline__ void rotate_tile(const RotateParams& P, int64_t tile, float2* turns) {
  constexpr int kGroups = kThreads / 8;
  const int head_tiles = (P.heads + P.tile_heads - 1) / P.tile_heads;
  const int64_t token0 = tile / head_tiles * P.tile_tokens;
  const int head0 = static_cast<int>(tile % head_tiles) * P.tile_heads;
  const int tokens = static_cast<int>(P.n_tokens - token0 < P.tile_tokens ? P.n_tokens - token0 : P.tile_tokens);
  const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
  const int tok = group % P.tile_tokens, step = kGroups / P.tile_tokens;
  const RowChunks c = row_chunks(P.r, l);
  const bool in_place = P.out == P.x;
  // what stays as it is needs no copy in place
  const bool on_a = c.turns_a || !in_place, on_b = c.turns_b || !in_place;
  const uint16_t* x = P.x + (token0 + tok) * P.x_st;
  uint16_t* out = P.out + (token0 + tok) * P.o_st;
  const int end = tok < tokens ? min(head0 + P.tile_heads, P.heads) : 0;
  uint4 a[kInFlight], b[kInFlight];
  const auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (h + i * step < end) {
        const uint4* from = reinterpret_cast<const uint4*>(x + (h + i * step) * P.x_sh);
        if (on_a) a[i] = from[c.a];
        if (on_b) b[i] = from[c.b];
      }
  };
  int h = head0 + group / P.tile_tokens;
  load(h);   // (on their way while the turns are computed)
  turns_to_shared<kThreads>(turns, P.r, P.positions, token0, tokens, P.transpose);
  if (h >= end) return;
  float2 cs[8];
  if (c.turns_a) lane_turns(cs, turns + tok * kMaxPairs, P.r, c);
  for (;;) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (h + i * step < end) {
        turn_chunks(a[i], b[i], cs, c, P.r.interleaved);
        uint4* to = reinterpret_cast<uint4*>(out + (h + i * step) * P.o_sh);
        if (on_a) to[c.a] = a[i];
        if (on_b) to[c.b] = b[i];
      }
    h += kInFlight * step;
    if (h >= end) return;
    load(h);
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
