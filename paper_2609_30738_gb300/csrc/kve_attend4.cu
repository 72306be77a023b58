// Attention over the paged 4-bit cache: rows (t, g) of a sequence and cache head h, the query heads h*G + g at
// positions len - T + t, over the visible tokens i < len - T + t + 1 of its pages, whose elements are s c + z with
// codes c in 0 .. 15 and two bf16 numbers a row:
//   l_i = (s_i (q . c_i) + z_i sum_j q_j) / sqrt(d),
//   out = sum_i softmax(l)_i s_i c_i + sum_i softmax(l)_i z_i,   lse = ln sum_i exp(l_i).
// Scales and zeros never touch a code: both products are of the codes alone.
//
// Bound by the read of the cache, 136 bytes a token and head. A code becomes a matrix operand in registers, with
// less than one instruction an element: the low four bits of an f16 are the subnormal c 2^-24 (and the next four
// 16 c 2^-24), so a word of eight codes is four operand registers by one shift and four masks, no conversion and
// nothing subtracted. The operands then have to be in registers (m16n8k16), where the loads put them:
//   S [rows][tokens]   = Q K^T     A = the query rows (f16, kept in registers), B = codes of a token, 32 a lane
//   O^T [d][rows]      = V^T W^T   A = codes of two tokens side by side, B = the weights where S left them
// The sums over d and over tokens do not care for the order of d and of tokens, as long as both operands have the
// same, so a lane's 16 bytes of K are eight k-steps as they lie, and a token's weight is already in the lane that
// holds the token's V codes. What the sums see of fewer than 32 bits:
//   q  bf16 times a power of two of its row, f16: exact down to 2^-31 of the row's largest (2^-27 in every second
//      element, whose codes are 16 times larger), an absolute 2^-38 of it below;
//   w  softmax(l)_i s_i over the row's largest such product so far, times 2^14, f16: 2^-12 of itself down to 2^-28 of
//      that largest, an absolute 2^-39 of it below.
// Maxima, sums, the part of z and the output are fp32. The reference of w is the product's own maximum, not the
// probability's, so that a token of far larger values costs the others nothing where it hardly counts.
//
// A warp takes 32 tokens a step from a ring of its own in shared memory that its lanes fill by 16-byte asynchronous
// copies, and has maxima, sums and output of its own: no warp waits for another before a part ends.
//
// The work is cut over the tokens like that of the 8-bit cache (kve_line.cuh): all tiles in one line, an even share
// for each CTA, whatever the lengths; a block of rows that falls to several CTAs is joined by the one that finishes
// last, from fp32 parts in token order.
#include "kve_internal.h"
#include "kve_line.cuh"
#include "kve_ptx.cuh"

namespace kve {
namespace {

constexpr int kStep = 32;                                  // tokens of a warp's step
constexpr int kRowBytes = kHeadDim / 2;                    // codes of a token
constexpr int kCodeBytes = kStep * kRowBytes;
constexpr int kParamBytes = kStep * 4;
constexpr int kStageBytes = 2 * (kCodeBytes + kParamBytes);

// R rows of a block, on W warps.
template <int R>
struct A4Cfg {
  static constexpr int kWarps = R == 8 ? 8 : 6;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kStages = R == 8 ? 3 : 4;
  static constexpr int kCtas = kAttend4Ctas;
  static constexpr int kRowWords = kHeadDim + 4;           // a row of a warp's output in shared memory
  static constexpr size_t kRing = size_t(kWarps) * kStages * kStageBytes;
  static constexpr size_t kMerge = size_t(kWarps) * R * kRowWords * sizeof(float);
  static constexpr size_t kSmem = kRing > kMerge ? kRing : kMerge;
};

template <int R>
struct A4Ctl {
  LineCtl<A4Cfg<R>::kWarps> line;
  float m[A4Cfg<R>::kWarps][R], l[A4Cfg<R>::kWarps][R];   // of the warps' rows, at the end of a part
  Block split[2];                                        // parts left for the join
  int last;
};

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

// 16 (or 4) bytes global -> shared, zeros where there is nothing to read (then src is not followed).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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

template <int R>
__global__ void __launch_bounds__(A4Cfg<R>::kThreads, A4Cfg<R>::kCtas)
cache_attend4_kernel(const __grid_constant__ AttendParams P) {
  using C = A4Cfg<R>;
  constexpr int W = C::kWarps, kThreads = C::kThreads, kHalves = R / 8;   // kHalves: rows of a lane
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ A4Ctl<R> ctl;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  // row / group, for groups that are no power of two as for those that are
  const auto row_token = [&](int row) {
    return P.group_inverse ? static_cast<int>(__umulhi(static_cast<uint32_t>(row), P.group_inverse)) : row;
  };
  const int rows = P.q_tokens * P.c.group;
  const int blocks = (rows + R - 1) / R;
  wait_previous_kernel();
  Cuts<kAttend4PartTiles> cuts;
  line_share<W>(P, blocks, kTileKeys, ctl.line, cuts);
  const int x0 = ctl.line.ends[0], x1 = ctl.line.ends[1];
  Block b = ctl.line.first;
  int splits = 0;
  const uint32_t ring = smem_u32(smem) + warp * (C::kStages * kStageBytes);
  const uint32_t* const kp = reinterpret_cast<const uint32_t*>(P.c.k_param);
  const uint32_t* const vp = reinterpret_cast<const uint32_t*>(P.c.v_param);
  // where this lane's copies go: token lane / 4 of 8, chunk lane % 4; the chunks of the tokens 4 .. 7 of every 8 change
  // places two by two, so that neither K's reads nor V's meet on a bank
  const uint32_t put = (lane >> 2) * kRowBytes + (((lane & 3) ^ ((lane >> 4) << 1)) << 4);
  // K: column n of an 8-token block is token n ^ (n >> 1 & 1), so that the two tokens of a lane's column pair are
  // neighbours of different parity
  const int ktok = g ^ (g >> 1 & 1);
  const uint32_t kget = ktok * kRowBytes + ((t ^ ((ktok >> 2) << 1)) << 4);
  // V: 8 bytes (g) of the tokens 2 t and 2 t + 1 of every 8, in the order of the columns
  const int odd = t & 1;
  const uint32_t vget = 2 * t * kRowBytes + (((g >> 1) ^ ((t >> 1) << 1)) << 4) + ((g & 1) << 3);
  const uint32_t vfirst = vget + odd * kRowBytes, vsecond = vget + (odd ^ 1) * kRowBytes;

  for (int x = x0; x < x1;) {
    const int end = min(x1, b.first + b.tiles);
    const int tok0 = (x - b.first) * kTileKeys, tok1 = min((end - b.first) * kTileKeys, b.len);
    const int steps = (tok1 - tok0 + kStep - 1) / kStep;
    const int first = steps * warp / W, last = steps * (warp + 1) / W;   // this warp's
    const float lb = len_bits(b.len);

    // ---------------------------------------------------------- the copies of a step
    const int32_t* const table = P.table + static_cast<int64_t>(b.r) * P.c.max_pages;
    const int shift = P.c.page_shift, page_mask = P.c.page - 1;
    // entries table_at .. table_at + 31 of the sequence's table, a lane each
    int table_at = (tok0 + first * kStep) >> shift, held = -1;
    const int pages = (b.len + page_mask) >> shift;
    const auto read_table = [&](int at) {
      table_at = at;
      held = at + lane < pages ? __ldg(table + at + lane) : -1;
      const bool outside = at + lane < pages && (held < 0 || held >= P.c.num_pages);
      if (outside) {
        atomicOr(P.err, kErrCheck);
        held = -1;
      }
    };
    uint32_t gaps = 0;   // bit k: step k of the ring has tokens that nobody sees
    const auto fetch = [&](int step, int slot) {
      const int at = tok0 + step * kStep;
      const int page0 = at >> shift, page1 = (at + kStep - 1) >> shift;
      if (page1 >= table_at + 32) read_table(page0);
      const int id0 = __shfl_sync(0xffffffffu, held, page0 - table_at), id1 = __shfl_sync(0xffffffffu, held, page1 - table_at);
      const uint32_t to = ring + slot * kStageBytes;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = at + 8 * i + (lane >> 2), id = i < 2 ? id0 : id1;
        const bool there = pos < b.len && id >= 0;
        const int64_t row = ((static_cast<int64_t>(max(id, 0)) * P.c.heads + b.h) << shift) + (pos & page_mask);
        const int64_t from = row * kRowBytes + (lane & 3) * 16;
        copy16(to + i * (8 * kRowBytes) + put, P.c.k + from, there);
        copy16(to + kCodeBytes + i * (8 * kRowBytes) + put, P.c.v + from, there);
      }
      {
        const int pos = at + lane, id = lane < 16 ? id0 : id1;
        const bool there = pos < b.len && id >= 0;
        const int64_t row = ((static_cast<int64_t>(max(id, 0)) * P.c.heads + b.h) << shift) + (pos & page_mask);
        copy4(to + 2 * kCodeBytes + lane * 4, kp + row, there);
        copy4(to + 2 * kCodeBytes + kParamBytes + lane * 4, vp + row, there);
      }
      gaps = (gaps & ~(1u << slot)) | (id0 < 0 || id1 < 0 || at + kStep > b.len ? 1u << slot : 0u);
    };
    if (first < last) read_table(table_at);
#pragma unroll
    for (int i = 0; i < C::kStages - 1; ++i) {
      if (first + i < last) fetch(first + i, i);
      copy_commit();
    }

    // ---------------------------------------------------------- the query rows
    uint32_t q[8][4];            // k-step, operand register
    float kq[kHalves], qb[kHalves];
    int seen[kHalves];
    long long out_row[kHalves];
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
      // 2^e brings the largest magnitude into [2^14, 2^15); elements beyond 2^112 make the row NaN
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
    float m[kHalves], top[kHalves], l[kHalves], z[kHalves];   // of logits; of logits + log2 s; sums of p and p z
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      m[e] = top[e] = -INFINITY;
      l[e] = z[e] = 0.f;
    }
    int slot = 0;
    for (int step = first; step < last; ++step) {
      copy_wait<C::kStages - 2>();
      __syncwarp();   // every lane's copies of this step have landed; the slot before this one has been read by all
      {
        const int next = step + C::kStages - 1, to = slot == 0 ? C::kStages - 1 : slot - 1;
        if (next < last) fetch(next, to);
        copy_commit();
      }
      const uint32_t at = ring + slot * kStageBytes;
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
      const int pos0 = tok0 + step * kStep;
      const bool some = (gaps >> slot & 1u) || (P.q_tokens > 1 && pos0 + kStep > b.len - P.q_tokens + 1);
      uint32_t hole = 0;   // pages outside the pool: bit 0 the first 16 tokens, bit 1 the others
      if (gaps >> slot & 1u) {
        const int id0 = (pos0 >> shift) < pages ? __ldg(table + (pos0 >> shift)) : 0;
        const int page1 = (pos0 + 16) >> shift;
        const int id1 = page1 < pages ? __ldg(table + page1) : 0;
        hole = (id0 < 0 || id0 >= P.c.num_pages ? 1u : 0u) | (id1 < 0 || id1 >= P.c.num_pages ? 2u : 0u);
      }
      // the four tokens' numbers: logits in place of the products
      float ls[4][2], vz[4][2];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const uint2 a = lds64(at + 2 * kCodeBytes + n * 32 + t * 8);
        const uint2 c = lds64(at + 2 * kCodeBytes + kParamBytes + n * 32 + t * 8);
        const uint32_t ka[2] = {odd ? a.y : a.x, odd ? a.x : a.y}, va[2] = {odd ? c.y : c.x, odd ? c.x : c.y};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          ls[n][j] = lg2(low_bf16(va[j]));
          vz[n][j] = high_bf16(va[j]);
#pragma unroll
          for (int e = 0; e < kHalves; ++e)
            s[n][2 * e + j] = fmaf(low_bf16(ka[j]), s[n][2 * e + j], high_bf16(ka[j]) * qb[e]) * kq[e];
        }
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
              if (gone || pos >= seen[e]) s[n][2 * e + j] = -INFINITY;
          }
      }
      uint32_t w[4][kHalves];
      bool moved = false;
      float back[kHalves];
#pragma unroll
      for (int e = 0; e < kHalves; ++e) {
        float mx = -INFINITY, tx = -INFINITY;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          mx = max3(mx, s[n][2 * e], s[n][2 * e + 1]);
          tx = max3(tx, s[n][2 * e] + ls[n][0], s[n][2 * e + 1] + ls[n][1]);
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        tx = fmaxf(tx, __shfl_xor_sync(0xffffffffu, tx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        tx = fmaxf(tx, __shfl_xor_sync(0xffffffffu, tx, 2));
        mx = fmaxf(mx, m[e]);
        tx = fmaxf(tx, top[e]);
        const float mr = (mx == -INFINITY ? 0.f : mx) + lb, tr = (tx == -INFINITY ? 0.f : tx);
        const float kept = ex2(m[e] - mr + lb);
        moved |= tx != top[e];
        back[e] = ex2(top[e] - tr);
        m[e] = mx;
        top[e] = tx;
        float ps = 0.f, pz = 0.f;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          float ww[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float xl = s[n][2 * e + j], p = ex2(xl - mr);
            ps += p;
            // (a NaN of a token that the row does not see stays out: some rows of the step may see it)
            pz = fmaf(p, some && xl == -INFINITY ? 0.f : vz[n][j], pz);
            ww[j] = some && xl == -INFINITY ? 0.f : ex2(xl + ls[n][j] - (tr - 14.f));
          }
          w[n][e] = f16x2(ww[0], ww[1]);
        }
        l[e] = fmaf(l[e], kept, ps);
        z[e] = fmaf(z[e], kept, pz);
      }
      if (__any_sync(0xffffffffu, moved)) {
        // factors of the rows 2 t and 2 t + 1 (whose columns of O^T this lane has)
#pragma unroll
        for (int e = 0; e < kHalves; ++e) {
          const float f0 = __shfl_sync(0xffffffffu, back[e], 8 * t), f1 = __shfl_sync(0xffffffffu, back[e], 8 * t + 4);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i][e][0] *= f0;
            o[i][e][1] *= f1;
            o[i][e][2] *= f0;
            o[i][e][3] *= f1;
          }
        }
      }
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
      slot = slot + 1 == C::kStages ? 0 : slot + 1;
    }
    copy_wait<0>();

    // ---------------------------------------------------------- the end of a part: the warps' rows together
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
      z[e] += __shfl_xor_sync(0xffffffffu, z[e], 1);
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
      z[e] += __shfl_xor_sync(0xffffffffu, z[e], 2);
    }
    __syncthreads();   // the rings are read; the sums before these are
    float* const mine = reinterpret_cast<float*>(smem) + warp * (R * C::kRowWords);
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
          v.x = fmaf(o[2 * i][e][j] * 256.f, ff, zz);
          v.y = fmaf(o[2 * i][e][2 + j] * 16.f, ff, zz);
          v.z = fmaf(o[2 * i + 1][e][j] * 256.f, ff, zz);
          v.w = fmaf(o[2 * i + 1][e][2 + j] * 16.f, ff, zz);
          *reinterpret_cast<float4*>(to + 4 * i) = v;
        }
      }
      if (t == 0) {
        ctl.m[warp][8 * e + g] = m[e];
        ctl.l[warp][8 * e + g] = l[e];
      }
    }
    __syncthreads();
    const bool whole = x == b.first && end == b.first + b.tiles;
    float* const part = P.partial + (static_cast<int64_t>(blockIdx.x) * 2 + (x == b.first)) * kAttend4PartWords;
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
        const float4 v = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (w * R + row) * C::kRowWords)[lane];
        sum = fmaf(ctl.l[w][row], f, sum);
        a.x = fmaf(v.x, f, a.x);
        a.y = fmaf(v.y, f, a.y);
        a.z = fmaf(v.z, f, a.z);
        a.w = fmaf(v.w, f, a.w);
      }
      if (whole) {
        emit_row(P, b, b.rb * R + row, rows, row_token, a, mx, sum, lb, lane);
      } else {
        reinterpret_cast<float4*>(part + row * kHeadDim)[lane] = a;
        if (lane == 0) {
          part[R * kHeadDim + row] = mx;
          part[R * kHeadDim + R + row] = sum;
        }
      }
    }
    if (!whole) {
      if (threadIdx.x == 0) ctl.split[splits] = b;
      ++splits;
    }
    __syncthreads();   // the rings may be filled again
    x = end;
    if (x < x1) next_block(P, blocks, kTileKeys, b);
  }

  // sequences without a token: their rows are zeros
  for (int r = blockIdx.x * W + warp; r < P.n_seq; r += W * gridDim.x)
    if (seq_len(P, r) == 0)
      for (int i = 0; i < P.q_tokens * P.c.hq; ++i) {
        const int64_t tok = static_cast<int64_t>(r) * P.q_tokens + i / P.c.hq;
        reinterpret_cast<uint2*>(P.out + tok * P.o_st + (i % P.c.hq) * P.o_sh)[lane] = make_uint2(0, 0);
        if (P.lse && lane == 0) P.lse[tok * P.c.hq + i % P.c.hq] = -INFINITY;
      }

  // ------------------------------------------------------------ the join of blocks that several CTAs had parts of
  allow_next_kernel();
  if (splits == 0) return;
  __threadfence();
  for (int k = 0; k < splits; ++k) {
    const Block s = ctl.split[k];
    int w0, w1;
    cuts.parts(s, &w0, &w1);
    __syncthreads();
    if (threadIdx.x == 0)
      ctl.last = inc_acq_rel_gpu(P.arrive + w0, static_cast<unsigned>(w1 - w0)) == static_cast<unsigned>(w1 - w0);
    __syncthreads();
    if (!ctl.last) continue;
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
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(C::kSmem));
  if (e != cudaSuccess) return e;
  // no more CTAs than there can be tiles
  const int64_t blocks = (p.q_tokens * p.c.group + R - 1) / R;
  const int64_t tiles = ((static_cast<int64_t>(p.c.max_pages) << p.c.page_shift) + kTileKeys - 1) / kTileKeys;
  const int64_t most = static_cast<int64_t>(C::kCtas) * c.sms;
  const int64_t want = tiles >= most ? most : tiles * p.n_seq * p.c.heads * blocks;
  return launch_after_previous(fn, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(C::kThreads), C::kSmem,
                               stream, p);
}

}  // namespace

cudaError_t launch_cache4_attend(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  return p.q_tokens * p.c.group <= 8 ? attend4_rows<8>(c, p, stream) : attend4_rows<16>(c, p, stream);
}

}  // namespace kve
