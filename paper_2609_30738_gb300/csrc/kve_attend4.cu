// Attention over the paged 4-bit cache: rows (t, g) of a sequence and cache head h, the query heads h*G + g at
// positions len - T + t, over the visible tokens i < len - T + t + 1 of its pages, whose elements are s c + z with
// codes c in 0 .. 15 and two bf16 numbers a row:
//   l_i = (s_i (q . c_i) + z_i sum_j q_j) / sqrt(d),
//   out = sum_i softmax(l)_i s_i c_i + sum_i softmax(l)_i z_i,   lse = ln sum_i exp(l_i).
// Scales and zeros never touch a code: both products are of the codes alone.
//
// Bound by the read of the cache, 136 bytes a token and head. A code becomes a matrix operand in registers, with
// about 0.7 instructions an element and no conversion: the low four bits of an f16 are the subnormal c 2^-24 (and the
// next four 16 c 2^-24), so a word of eight codes is four operand registers by one shift and four masks. The operands then
// have to be in registers (mma.sync m16n8k16), where the loads put them:
//   S [rows][tokens]   = Q K^T     A = the query rows (f16, kept in registers), B = codes of a token, 32 a lane
//   O^T [d][rows]      = V^T W^T   A = codes of two tokens side by side, B = the weights where S left them
// The sums over d and over tokens do not care for the order of d and of tokens, as long as both operands have the
// same, so a lane's 16 bytes of K are eight k-steps as they lie, and a token's weight is already in the lane that
// holds the token's V codes. What the sums see of fewer than 32 bits:
//   q  bf16 times a power of two of its row, f16: exact down to 2^-31 of the row's largest (2^-27 in every second
//      element, whose codes are 16 times larger), an absolute 2^-38 of it below;
//   w  softmax(l)_i s_i over a reference within 2^8 of the row's largest such product so far, times 2^6, f16: 2^-12 of
//      itself down to 2^-20 of that reference, an absolute 2^-31 of it below.
// Maxima, sums, the part of z and the output are fp32. The reference of w is the product's own, not the probability's, so
// that a token of far larger values costs the others nothing where it hardly counts. References move only when a maximum
// passes them by 2^8, which leaves the rescaling of the output to a few steps.
//
// A consumer warp takes 32 tokens a step from a ring of its own in shared memory (TMA boxes of 32 rows with the 64-byte
// swizzle), and has maxima, sums and output of its own: no warp waits for another before a part ends. One warp fills all
// rings, a lane for each, across the ends of parts.
//
// The work is cut over the tokens like that of the 8-bit cache (kve_line.cuh): all tiles in one line, an even share
// for each CTA, whatever the lengths; a block of rows that falls to several CTAs is joined by the one that finishes
// last, from fp32 parts in token order.
#include <type_traits>

#include "kve_internal.h"
#include "kve_line.cuh"
#include "kve_ptx.cuh"

namespace kve {
namespace {

constexpr int kStep = 32;                                  // tokens of a warp's step
constexpr int kRowBytes = kHeadDim / 2;                    // codes of a token
constexpr int kCodeBytes = kStep * kRowBytes;
constexpr int kStageBytes = 2 * kCodeBytes;                // K, then V

// R rows of a block, on W consumer warps (and one that copies).
template <int R>
struct A4Cfg {
  static constexpr int kWarps = R == 8 ? 7 : 11;
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kStages = 2;
  static constexpr int kCtas = R == 8 ? kAttend4Ctas : 1;
  static constexpr int kRowWords = kHeadDim + 4;           // a row of a warp's output in shared memory
  static constexpr size_t kMerge = size_t(kWarps) * kStages * kStageBytes;
  static constexpr size_t kCtl = kMerge + size_t(kWarps) * R * kRowWords * sizeof(float);
};

// A part, tiles x .. end - 1 of block b, from token tok0 of its sequence on; steps first .. last - 1 of it are a warp's.
struct Part {
  Block b;
  int x, end, tok0, first, last;
  template <int W>
  __device__ __forceinline__ void set(int x1, int warp) {
    end = min(x1, b.first + b.tiles);
    tok0 = (x - b.first) * kTileKeys;
    const int steps = (min((end - b.first) * kTileKeys, b.len) - tok0 + kStep - 1) / kStep;
    first = steps * warp / W;
    last = steps * (warp + 1) / W;
  }
};

template <int R>
struct A4Ctl {
  static constexpr int W = A4Cfg<R>::kWarps, S = A4Cfg<R>::kStages;
  alignas(128) uint32_t param[W][S][2][kStep];   // K's, V's
  float4 tokens[W][kStep];                       // of a step's tokens: K's s and z, V's log2 s and z
  uint64_t full[W][S], empty[W][S];
  uint32_t holes[W][S];                          // pages outside the pool: bit 0 of the first 16 tokens, bit 1 of the others
  LineCtl<W + 1> line;
  Part part[W];                                  // (all lanes write the same)
  float m[W][R], l[W][R];                        // of the warps' rows, at the end of a part
  Block split[2];                                // parts left for the join
  int last[2];                                   // whether this CTA joins them
  int abort, never;                              // never: stays 0 (waits that a given-up call still has to make)
};

// How far (log2) a row's largest product passes its reference before that moves. Weights count from 2^(14 - kLazy) there.
constexpr float kLazy = 8.f;

template <int R>
constexpr size_t attend4_smem() {
  return A4Cfg<R>::kCtl + sizeof(A4Ctl<R>);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ float low_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// log2 of the unit in which a row's probabilities are summed: then a sum of values near bf16's largest passes that as
// little as the probabilities' sum passes 1.
__device__ __forceinline__ float len_bits(int len) { return static_cast<float>(32 - __clz(len - 1)); }   // (1: 0)

static_assert(attend4_smem<8>() <= 113 * 1024 && attend4_smem<16>() <= 227 * 1024, "two CTAs an SM, or one");

// A barrier of the consumer warps, and whether any of their threads says so.
template <int kThreads>
__device__ __forceinline__ bool meet_or(bool x) {
  uint32_t any;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(any)
               : "r"(x ? 1u : 0u), "n"(kThreads)
               : "memory");
  return any != 0;
}

template <int R>
__global__ void __launch_bounds__(A4Cfg<R>::kThreads, A4Cfg<R>::kCtas)
cache_attend4_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const __grid_constant__ AttendParams P) {
  using C = A4Cfg<R>;
  constexpr int W = C::kWarps, kHalves = R / 8;   // kHalves: rows of a lane
  constexpr int S = C::kStages;
  extern __shared__ __align__(1024) uint8_t smem[];   // the swizzle counts from 512 bytes
  A4Ctl<R>& ctl = *reinterpret_cast<A4Ctl<R>*>(smem + C::kCtl);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows = P.q_tokens * P.c.group;
  const int blocks = (rows + R - 1) / R;
  if (warp < W && lane == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&ctl.full[warp][i], 1);
      mbar_init(&ctl.empty[warp][i], 1);
    }
    fence_mbar_init();
  }
  if (threadIdx.x == 0) {
    ctl.abort = ctl.never = 0;
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  wait_previous_kernel();
  Cuts<kAttend4PartTiles> cuts;
  line_share<W + 1>(P, blocks, kTileKeys, ctl.line, cuts);
  const int x0 = ctl.line.ends[0], x1 = ctl.line.ends[1];
  const int shift = P.c.page_shift;
  const auto fail = [&]() {
    ctl.abort = 1;
    atomicOr(P.err, kErrWait);
  };

  if (warp == W) {
    // ------------------------------------------------------------ copies: lane w fills the ring of warp w
    bool more = lane < W && x0 < x1;
    Part a;
    a.b = ctl.line.first;
    a.x = x0;
    int step = 0, at = 0, head = 0, id0 = -1, id1 = -1;   // the next copies: first token, first row of the head in a page, pages
    const auto page = [&](int token) {
      if (token >= a.b.len) return 0;   // (nobody sees what is there)
      return __ldg(P.table + static_cast<int64_t>(a.b.r) * P.c.max_pages + (token >> shift));
    };
    const auto valid = [&](int id) { return id >= 0 && id < P.c.num_pages; };
    const auto advance = [&]() {   // to the step behind `step - 1`, in this part or a later one
      while (step >= a.last) {
        a.x = a.end;
        if (a.x >= x1) {
          more = false;
          return;
        }
        next_block(P, blocks, kTileKeys, a.b);
        a.template set<W>(x1, lane);
        step = a.first;
      }
      at = a.tok0 + step * kStep;
      head = a.b.h << shift;
      id0 = page(at);
      if (P.c.page < kStep) id1 = page(at + 16);   // (looked at when the copies are made, a turn later)
    };
    if (more) {
      a.template set<W>(x1, lane);
      step = a.first;
      advance();
    }
    // Pages of a call that reads more than L2 keeps leave it first.
    const uint64_t policy = x1 - x0 > 8 ? l2_policy_evict_first() : l2_policy_evict_normal();
    const int rows0 = min(P.c.page, kStep);   // boxes of 32 rows, or of a page's 16
    uint32_t fetched = 0;
    uint64_t since = global_timer_ns();
    bool stuck = false;
    while (__any_sync(0xffffffffu, more)) {
      const uint32_t slot = fetched % S;
      const bool go = more && (fetched < S || mbar_test_wait(&ctl.empty[lane][slot], (fetched / S & 1) ^ 1));
      if (go) {
        uint64_t* bar = &ctl.full[lane][slot];
        const bool ok0 = valid(id0), ok1 = rows0 < kStep ? valid(id1) : ok0;
        ctl.holes[lane][slot] = (ok0 ? 0u : 1u) | (ok1 ? 0u : 2u);
        if (!ok0 || !ok1) atomicOr(P.err, kErrCheck);
        mbar_arrive_expect_tx(bar, ((ok0 ? rows0 : 0) + (rows0 < kStep && ok1 ? rows0 : 0)) * (2 * (kRowBytes + 4)));
        for (int i = 0; i < kStep; i += rows0) {
          const int id = i == 0 ? id0 : id1;
          if (!(i == 0 ? ok0 : ok1)) continue;
          const int row = (id * P.c.heads << shift) + head + ((at + i) & (P.c.page - 1));
          uint8_t* to = smem + (lane * S + slot) * kStageBytes + i * kRowBytes;
          tma_load_2d_hint(to, &tm_k, 0, row, bar, policy);
          tma_load_2d_hint(to + kCodeBytes, &tm_v, 0, row, bar, policy);
          bulk_load(&ctl.param[lane][slot][0][i], P.c.k_param + row, rows0 * 4, bar);
          bulk_load(&ctl.param[lane][slot][1][i], P.c.v_param + row, rows0 * 4, bar);
        }
        ++fetched;
        ++step;
        advance();
      }
      if (__any_sync(0xffffffffu, go)) {
        since = global_timer_ns();
      } else {
        __nanosleep(32);
        stuck = *static_cast<volatile int*>(&ctl.abort) != 0 || global_timer_ns() - since > P.wait_limit_ns;
        if (__any_sync(0xffffffffu, stuck)) break;
      }
    }
    if (__any_sync(0xffffffffu, stuck)) {
      // a wait ran out: the copies in flight end before the shared memory does
      if (lane == 0) fail();
      for (int w = 0; w < W; ++w) {
        const uint32_t n = __shfl_sync(0xffffffffu, fetched, w);
        for (uint32_t k = n > S ? n - S : 0; k < n; ++k)
          warp_wait(&ctl.full[w][k % S], (k / S) & 1, P.wait_limit_ns, &ctl.never);
      }
    }
    // sequences without a token: their rows are zeros
    for (int r = blockIdx.x; r < P.n_seq; r += gridDim.x)
      if (seq_len(P, r) == 0)
        for (int i = 0; i < P.q_tokens * P.c.hq; ++i) {
          const int64_t tok = static_cast<int64_t>(r) * P.q_tokens + i / P.c.hq;
          reinterpret_cast<uint2*>(P.out + tok * P.o_st + (i % P.c.hq) * P.o_sh)[lane] = make_uint2(0, 0);
          if (P.lse && lane == 0) P.lse[tok * P.c.hq + i % P.c.hq] = -INFINITY;
        }
    allow_next_kernel();
    return;
  }

  // -------------------------------------------------------------- the consumers
  const int g = lane >> 2, t = lane & 3;
  // row / group, for groups that are no power of two as for those that are
  const auto row_token = [&](int row) {
    return P.group_inverse ? static_cast<int>(__umulhi(static_cast<uint32_t>(row), P.group_inverse)) : row;
  };
  int splits = 0;
  const uint32_t ring = smem_u32(smem) + warp * (S * kStageBytes);
  // K: column n of an 8-token block is token n ^ (n >> 1 & 1), so that the two tokens of a lane's column pair are
  // neighbours of different parity: with the swizzle (a 16-byte chunk c of row r lies at c ^ (r >> 1 & 3)) neither K's reads nor
  // V's meet on a bank
  const int ktok = g ^ (g >> 1 & 1);
  const uint32_t kget = ktok * kRowBytes + ((t ^ (ktok >> 1)) << 4);
  // V: 8 bytes (g) of the tokens 2 t and 2 t + 1 of every 8, in the order of the columns
  const int odd = t & 1;
  const uint32_t vget = 2 * t * kRowBytes + (((g >> 1) ^ t) << 4) + ((g & 1) << 3);
  const uint32_t vfirst = vget + odd * kRowBytes, vsecond = vget + (odd ^ 1) * kRowBytes;
  const float4* const numbers = ctl.tokens[warp] + 2 * t;   // of token 2 t + (j ^ odd) of every 8
  uint32_t used = 0;
  bool ok = true, failed = false;
  if (x0 < x1) {
    Part a;
    a.b = ctl.line.first;
    a.x = x0;
    a.template set<W>(x1, warp);
    ctl.part[warp] = a;
    __syncwarp();
  }
  for (int x = x0; x < x1;) {
    const Part& part = ctl.part[warp];
    const Block& b = part.b;
    const float lb = len_bits(b.len);
    // ---------------------------------------------------------- the query rows
    uint32_t q[8][4];            // k-step, operand register
    float kq[kHalves], qb[kHalves];
    int seen[kHalves];
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      const int row = b.rb * R + 8 * e + g;
      const int qt = row_token(row), hq = b.h * P.c.group + row - qt * P.c.group;
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = make_uint4(0, 0, 0, 0);
      if (row < rows) {
        const uint16_t* from = P.q + (static_cast<int64_t>(b.r) * P.q_tokens + qt) * P.q_st + hq * P.q_sh + 32 * t;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __ldg(reinterpret_cast<const uint4*>(from) + i);
      }
      seen[e] = row < rows ? b.len - P.q_tokens + qt + 1 : 0;
      const uint32_t* u = &v[0].x;
      uint32_t most = 0;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        most = max(most, max(u[i] << 16 & 0x7fff0000u, u[i] & 0x7fff0000u));
        sum += low_bf16(u[i]) + high_bf16(u[i]);
      }
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      // 2^up brings the largest magnitude into [2^14, 2^15); one of 2^112 or more, or a NaN, makes the row NaN
      const int ex = static_cast<int>(most >> 23);
      const int up = min(14 + 127 - ex, 126);
      const float scale = __uint_as_float(static_cast<uint32_t>(up + 127) << 23);
      kq[e] = P.alpha * __uint_as_float(static_cast<uint32_t>(min(24 - up, 127) + 127) << 23);
      qb[e] = ex >= 127 + 112 ? __uint_as_float(0x7fc00000u) : sum * scale * 5.9604644775390625e-8f;   // 2^-24
#pragma unroll
      for (int w = 0; w < 4; ++w) {   // 8 elements: n and n + 4 go together
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[2 * i] = low_bf16(u[4 * w + i]) * scale;
          f[2 * i + 1] = high_bf16(u[4 * w + i]) * scale;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          q[2 * w + h][e] = f16x2(f[2 * h], f[2 * h + 4]);
          q[2 * w + h][2 + e] = f16x2(f[2 * h + 1] * 0.0625f, f[2 * h + 5] * 0.0625f);
        }
      }
    }
    if constexpr (kHalves == 1) {
#pragma unroll
      for (int k = 0; k < 8; ++k) q[k][1] = q[k][3] = 0;
    }

    // ---------------------------------------------------------- the steps
    float o[8][kHalves][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < kHalves; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][e][k] = 0.f;
    float m[kHalves], top[kHalves], l[kHalves], z[kHalves];   // the lane's maximum; the row's reference; the lane's sums of p, p z
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      m[e] = top[e] = -INFINITY;
      l[e] = z[e] = 0.f;
    }
    const int last = part.last, tok0 = part.tok0, all_see = b.len - P.q_tokens + 1;
#pragma unroll 1
    for (int step = part.first; step < last; ++step) {
      const uint32_t slot = used % S;
      if (!warp_wait(&ctl.full[warp][slot], (used / S) & 1, P.wait_limit_ns, &ctl.abort)) {
        ok = false;
        break;
      }
      ++used;
      const uint32_t at = ring + slot * kStageBytes;
      {
        // a lane a token: its four numbers for every lane
        const uint32_t a = ctl.param[warp][slot][0][lane], c = ctl.param[warp][slot][1][lane];
        ctl.tokens[warp][lane] = make_float4(low_bf16(a), high_bf16(a), lg2(low_bf16(c)), high_bf16(c));
      }
      float s[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) s[n][k] = 0.f;
        const uint4 v = lds128(at + n * (8 * kRowBytes) + kget);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t hi = u[w] >> 8;
          mma_f16(s[n], q[2 * w], u[w] & 0x000f000fu, u[w] & 0x00f000f0u);
          mma_f16(s[n], q[2 * w + 1], hi & 0x000f000fu, hi & 0x00f000f0u);
        }
      }
      __syncwarp();
      const int pos0 = tok0 + step * kStep;
      const uint32_t hole = ctl.holes[warp][slot];
      const bool some = hole != 0 || pos0 + kStep > all_see;   // tokens that not all rows see
      // logits (over kq) in place of the products; beside them their sums with the log2 of V's s, or for two rows a lane
      // that alone (registers)
      float beside[4][2] = {};
      const auto with_s = [&](int n, int j, int e) {
        return kHalves == 1 ? beside[n][j] : fmaf(s[n][2 * e + j], kq[e], beside[n][j]);
      };
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float4 f = numbers[8 * n + (j ^ odd)];
#pragma unroll
          for (int e = 0; e < kHalves; ++e) s[n][2 * e + j] = fmaf(f.x, s[n][2 * e + j], f.y * qb[e]);
          beside[n][j] = kHalves == 1 ? fmaf(s[n][j], kq[0], f.z) : f.z;
        }
      if (some) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int pos = pos0 + 8 * n + 2 * t + (j ^ odd);
            const bool gone = hole >> (n >> 1) & 1u;
#pragma unroll
            for (int e = 0; e < kHalves; ++e)
              if (gone || pos >= seen[e]) {
                s[n][2 * e + j] = -INFINITY;
                if (kHalves == 1) beside[n][j] = -INFINITY;
              }
          }
      }
      // the lane's own largest logits, and the row's references of the products within 2^kLazy of the largest so far
      float tx[kHalves];
      bool moved = false;
#pragma unroll
      for (int e = 0; e < kHalves; ++e) {
        float mx = -INFINITY;
        tx[e] = -INFINITY;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          mx = max3(mx, s[n][2 * e], s[n][2 * e + 1]);
          tx[e] = max3(tx[e], with_s(n, 0, e), with_s(n, 1, e));
        }
        mx = fmaxf(mx * kq[e], m[e]);
        const float kept = ex2(m[e] - (mx == -INFINITY ? 0.f : mx));
        m[e] = mx;
        l[e] *= kept;
        z[e] *= kept;
        moved |= tx[e] > top[e] + kLazy;
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int e = 0; e < kHalves; ++e) {
          tx[e] = fmaxf(tx[e], __shfl_xor_sync(0xffffffffu, tx[e], 1));
          tx[e] = fmaxf(fmaxf(tx[e], __shfl_xor_sync(0xffffffffu, tx[e], 2)), top[e]);
          const float back = ex2(top[e] - (tx[e] == -INFINITY ? 0.f : tx[e]));
          top[e] = tx[e];
          // factors of the rows 2 t and 2 t + 1 (whose columns of O^T this lane has)
          const float f0 = __shfl_sync(0xffffffffu, back, 8 * t), f1 = __shfl_sync(0xffffffffu, back, 8 * t + 4);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i][e][0] *= f0;
            o[i][e][1] *= f1;
            o[i][e][2] *= f0;
            o[i][e][3] *= f1;
          }
        }
      }
      uint32_t w[4][kHalves];
      const auto weigh = [&](auto kSome) {
#pragma unroll
        for (int e = 0; e < kHalves; ++e) {
          const float mr = (m[e] == -INFINITY ? 0.f : m[e]) + lb, tr = (top[e] == -INFINITY ? 0.f : top[e]) - (14.f - kLazy);
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            float ww[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float p = ex2(fmaf(s[n][2 * e + j], kq[e], -mr));
              // (a NaN of a token that the row does not see stays out: some rows of the step may see it)
              const bool out = kSome.value && s[n][2 * e + j] == -INFINITY;
              l[e] += p;
              z[e] = fmaf(p, out ? 0.f : numbers[8 * n + (j ^ odd)].w, z[e]);
              ww[j] = out && kHalves > 1 ? 0.f : ex2(with_s(n, j, e) - tr);
            }
            w[n][e] = f16x2(ww[0], ww[1]);
          }
        }
      };
      if (some)
        weigh(std::true_type{});
      else
        weigh(std::false_type{});
#pragma unroll
      for (int n = 0; n < 4; n += 2) {
        const uint32_t va = at + kCodeBytes + n * (8 * kRowBytes);
        const uint2 a0 = lds64(va + vfirst), a1 = lds64(va + vsecond);
        const uint2 b0 = lds64(va + 8 * kRowBytes + vfirst), b1 = lds64(va + 8 * kRowBytes + vsecond);
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // four of a word's codes of both tokens side by side
          const uint32_t sel = i & 1 ? 0x7632u : 0x5410u;
          const uint32_t p0 = __byte_perm(i & 2 ? a0.y : a0.x, i & 2 ? a1.y : a1.x, sel);
          const uint32_t p1 = __byte_perm(i & 2 ? b0.y : b0.x, i & 2 ? b1.y : b1.x, sel);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t c0 = h ? p0 >> 8 : p0, c1 = h ? p1 >> 8 : p1;
            const uint32_t a[4] = {c0 & 0x000f000fu, c0 & 0x00f000f0u, c1 & 0x000f000fu, c1 & 0x00f000f0u};
#pragma unroll
            for (int e = 0; e < kHalves; ++e) mma_f16(o[2 * i + h][e], a, w[n][e], w[n + 1][e]);
          }
        }
      }
      __syncwarp();   // the stage and the tokens' numbers have been read
      if (lane == 0) mbar_arrive(&ctl.empty[warp][slot]);
    }
    if (!ok && lane == 0) fail();

    // ---------------------------------------------------------- the end of a part: the warps' rows together
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      const float mine = m[e];
      m[e] = fmaxf(m[e], __shfl_xor_sync(0xffffffffu, m[e], 1));
      m[e] = fmaxf(m[e], __shfl_xor_sync(0xffffffffu, m[e], 2));
      const float kept = ex2(mine - (m[e] == -INFINITY ? 0.f : m[e]));
      l[e] *= kept;
      z[e] *= kept;
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
      z[e] += __shfl_xor_sync(0xffffffffu, z[e], 1);
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
      z[e] += __shfl_xor_sync(0xffffffffu, z[e], 2);
    }
    meet_or<32 * W>(false);   // the sums of the part before are read
    float* const merge = reinterpret_cast<float*>(smem + C::kMerge);
    float* const mine = merge + warp * (R * C::kRowWords);
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      // quarters of sum p (s c + z), so that neither term alone passes the largest float
      const float f = ex2((top[e] == -INFINITY ? 0.f : top[e]) - (m[e] == -INFINITY ? 0.f : m[e]) - lb);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int from = 8 * t + 4 * j;
        const float ff = __shfl_sync(0xffffffffu, f, from), zz = 0.25f * __shfl_sync(0xffffffffu, z[e], from);
        float* to = mine + (8 * e + 2 * t + j) * C::kRowWords + 16 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float4 v;
          // (c 2^-24 or 16 c 2^-24, weights times 2^(14 - kLazy), a quarter)
          v.x = fmaf(o[2 * i][e][j] * 65536.f, ff, zz);
          v.y = fmaf(o[2 * i][e][2 + j] * 4096.f, ff, zz);
          v.z = fmaf(o[2 * i + 1][e][j] * 65536.f, ff, zz);
          v.w = fmaf(o[2 * i + 1][e][2 + j] * 4096.f, ff, zz);
          *reinterpret_cast<float4*>(to + 4 * i) = v;
        }
      }
      if (t == 0) {
        ctl.m[warp][8 * e + g] = m[e];
        ctl.l[warp][8 * e + g] = l[e];
      }
    }
    failed = meet_or<32 * W>(!ok);
    if (failed) break;
    const bool whole = x == b.first && part.end == b.first + b.tiles;
    float* const out = P.partial + (static_cast<int64_t>(blockIdx.x) * 2 + (x == b.first)) * kAttend4PartWords;
    for (int row = warp; row < R; row += W) {
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) mx = fmaxf(mx, ctl.m[w][row]);
      const float mr = mx == -INFINITY ? 0.f : mx;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = ex2(ctl.m[w][row] - mr);
        const float4 v = reinterpret_cast<const float4*>(merge + (w * R + row) * C::kRowWords)[lane];
        sum = fmaf(ctl.l[w][row], f, sum);
        a.x = fmaf(v.x, f, a.x);
        a.y = fmaf(v.y, f, a.y);
        a.z = fmaf(v.z, f, a.z);
        a.w = fmaf(v.w, f, a.w);
      }
      if (whole) {
        emit_row(P, b, b.rb * R + row, rows, row_token, a, mx, sum, lb, lane);
      } else {
        reinterpret_cast<float4*>(out + row * kHeadDim)[lane] = a;
        if (lane == 0) {
          out[R * kHeadDim + row] = mx;
          out[R * kHeadDim + R + row] = sum;
        }
      }
    }
    if (!whole) {
      if (threadIdx.x == 0) ctl.split[splits] = b;
      ++splits;
    }
    x = part.end;
    if (x < x1) {
      Part a = part;
      a.x = x;
      next_block(P, blocks, kTileKeys, a.b);
      a.template set<W>(x1, warp);
      __syncwarp();
      ctl.part[warp] = a;
      __syncwarp();
    }
  }
  if (failed) return;

  // ------------------------------------------------------------ the join of blocks that several CTAs had parts of
  allow_next_kernel();
  if (splits == 0) return;
  __threadfence();
  meet_or<32 * W>(false);   // every thread's part of the sums is out, and ctl.split is written
  for (int k = 0; k < splits; ++k) {
    const Block s = ctl.split[k];
    int w0, w1;
    cuts.parts(s, &w0, &w1);
    if (threadIdx.x == 0)
      ctl.last[k] = inc_acq_rel_gpu(P.arrive + w0, static_cast<unsigned>(w1 - w0)) == static_cast<unsigned>(w1 - w0);
    meet_or<32 * W>(false);
    if (!ctl.last[k]) continue;
    __threadfence();
    const int parts = w1 - w0 + 1;
    const float lb = len_bits(s.len);
    for (int row = warp; row < R && s.rb * R + row < rows; row += W) {
      // part p: slot 0 of CTA w0 + p, of the first one slot 1
      const auto at = [&](int p) { return P.partial + (static_cast<int64_t>(w0 + p) * 2 + (p == 0)) * kAttend4PartWords; };
      float mx = -INFINITY;
      for (int p = lane; p < parts; p += 32) mx = fmaxf(mx, __ldcg(at(p) + R * kHeadDim + row));
      mx = warp_max(mx);
      const float mr = mx == -INFINITY ? 0.f : mx;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll 8
      for (int p = 0; p < parts; ++p) {
        const float* from = at(p);
        const float f = ex2(__ldcg(from + R * kHeadDim + row) - mr);
        const float4 v = __ldcg(reinterpret_cast<const float4*>(from + row * kHeadDim) + lane);
        sum = fmaf(__ldcg(from + R * kHeadDim + R + row), f, sum);
        a.x = fmaf(v.x, f, a.x);
        a.y = fmaf(v.y, f, a.y);
        a.z = fmaf(v.z, f, a.z);
        a.w = fmaf(v.w, f, a.w);
      }
      emit_row(P, s, s.rb * R + row, rows, row_token, a, mx, sum, lb, lane);
    }
  }
}

template <int R>
cudaError_t attend4_rows(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  using C = A4Cfg<R>;
  auto* fn = cache_attend4_kernel<R>;
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(attend4_smem<R>()));
  if (e != cudaSuccess) return e;
  // no more CTAs than there can be tiles
  const int64_t blocks = (p.q_tokens * p.c.group + R - 1) / R;
  const int64_t tiles = ((static_cast<int64_t>(p.c.max_pages) << p.c.page_shift) + kTileKeys - 1) / kTileKeys;
  const int64_t most = static_cast<int64_t>(C::kCtas) * c.sms;
  const int64_t want = tiles >= most ? most : tiles * p.n_seq * p.c.heads * blocks;
  return launch_after_previous(fn, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(C::kThreads),
                               attend4_smem<R>(), stream, c.tm_k, c.tm_v, p);
}

}  // namespace

cudaError_t launch_cache4_attend(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  return p.q_tokens * p.c.group <= 8 ? attend4_rows<8>(c, p, stream) : attend4_rows<16>(c, p, stream);
}

}  // namespace kve
