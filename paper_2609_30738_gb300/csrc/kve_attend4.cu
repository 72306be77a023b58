// Attention over the paged 4-bit cache: rows (t, g) of a sequence and cache head h, the query heads h*G + g at
// positions len - T + t, over the visible tokens i < len - T + t + 1 of its pages, whose elements are s c + z with
// codes c in 0 .. 15 and two bf16 numbers a row:
//   l_i = (s_i (q . c_i) + z_i sum_j q_j) / sqrt(d),
//   out = sum_i softmax(l)_i s_i c_i + sum_i softmax(l)_i z_i,   lse = ln sum_i exp(l_i).
// Scales and zeros never touch a code: both products are of the codes alone.
//
// Bound by the read of the cache, 136 bytes a token and head, and by start and end: 64 ragged sequences of 512 to 16384 tokens and 8
// heads (237 MB) take 47.2 us where a copy's rate is 35.5, and 400 of 100 to 8000 (759 MB) 131, so between the two it runs at 93% of
// that rate, beside 9 us. 5 of them are any call's (96 tokens: lengths, cut, table, first codes, a step, output); then the first copies
// of all CTAs at once, the ends of parts, the join, which is longest for few heads of long sequences (one of 131072 tokens, 143 MB, 33.3
// of 21.3). A step of a warp, 32 tokens and 8 rows, is 375 instructions, half of them the integer unit's, most of which unpack codes.
// 16 rows are 494, of them 64 matrix products, and two warps a scheduler that wait for their own results: 24 sequences of 500 to 8192
// tokens 29.2 us of 10, 16 of 8192 with 32 rows 76 of 21.7.
//
// A code becomes a matrix operand in registers, with half an instruction an element and no conversion: the low four bits of an f16
// are the subnormal c 2^-24 and the next four 16 c 2^-24, so a word of eight codes is four operand registers by a shift and masks. The
// operands then have to be in registers (mma.sync m16n8k16; in e4m3 that instruction is made of conversions and the f16 one here:
// 131072 tokens 50.5 us for 40.8 at the time), where the loads put them:
//   S^T [tokens][rows] = K Q^T     A = codes of two tokens, 32 a lane and token, B = the query rows (f16, from shared memory)
//   O^T [d][rows]      = V^T W^T   A = codes of two tokens side by side (transposing matrix loads), B = the weights,
//                                  S^T's registers after an 8 x 8 transposition
// so 8 rows fill the N side (tokens there instead took 66.3 us for 61.2 on the 64). The sums over d do not care for its order, as long
// as both operands have the same, so a lane's 16 bytes of K are eight k-steps as they lie. V's second codes stay with the first ones,
// c + 16 c', which saves a mask, and the end takes the first one's sum out again: both are fp32 sums of exact products, and the
// difference is off by 16 / 15 of what the sum of 16 c' alone would be. What the sums see of fewer than 32 bits:
//   q  bf16 times a power of two of its row, f16: exact down to 2^-31 of the row's largest (2^-27 in every second
//      element, whose codes are 16 times larger), an absolute 2^-35 of it below;
//   w  softmax(l)_i s_i over a reference within 2^8 of the row's largest such product so far, times 2^6, f16: 2^-12 of
//      itself down to 2^-20 of that reference, an absolute 2^-31 of it below.
// Maxima, sums, the part of z and the output are fp32. The reference of w is the product's own, not the probability's, so
// that a token of far larger values costs the others nothing where it hardly counts. References move only when a maximum
// passes them by 2^8, which leaves the rescaling of the output to a few steps. What a warp leaves at the end of a
// part, and a CTA for the join, is the average over its tokens beside their maximum and sum, so values at either end of fp32 keep their
// bits whatever the length; the sum of p z before that is scaled down by the length only once a |z| of 2^96 comes. (Sums in a unit of the length throughout lose s near
// 2^-119 behind some thousand tokens; they took 46.9 us for 47.2 on the 64, 33.0 for 33.3 and 74.6 for 76.)
//
// A warp takes 32 tokens a step from a ring of its own in shared memory, and has maxima, sums and output of its own: no warp waits for
// another before a part ends. It fills its ring itself, across the ends of parts, by asynchronous copies that stand between its
// products, with as few instructions as will do: a tenth of them was 2 us of the 64. (A tensor copy holds its warp for more than 100
// cycles, and a step is four of them, with pages of 16 eight: 131072 tokens took 40.9 us for 38.2; one warp that fills all rings 40.8 for
// 38.6. The next step's scores between the products with V 36.2 for 35.3, their registers.)
//
// The work is cut over the tokens like that of the 8-bit cache (kve_line.cuh): all tiles in one line, an even share
// for each CTA, whatever the lengths; a block of rows that falls to several CTAs is joined by the one that finishes
// last, from fp32 parts in token order.
#include <climits>
#include <type_traits>

#include "kve_internal.h"
#include "kve_line.cuh"
#include "kve_ptx.cuh"

namespace kve {
namespace {

constexpr int kStep = 32;                                  // tokens of a warp's step
constexpr int kRowBytes = kHeadDim / 2;                    // codes of a token
constexpr int kCodeBytes = kStep * kRowBytes;
constexpr int kNumbers = 2 * kCodeBytes;                   // K, V, then the numbers of K's rows and of V's
constexpr int kStageBytes = kNumbers + 2 * kStep * 4;

// R rows of a block on W warps of a CTA (attend4_rows). 12 warps an SM for 8 rows, or one CTA of 8, and 8 for 16: registers that let
// a warp's own instructions overlap are worth more than warps. (16 warps of 128 registers: 64 ragged sequences 50.6 us for 46.9, 8 warps
// and 4 stages 60.5. 16 rows with 12 warps, 168 registers and spills: 24 sequences of 4 drafts 33.5 for 29.0, with 16 warps 64.) A ring of 4 stages
// instead of 3 took 48.2 and 29.9.
template <int R, int W>
struct A4Cfg {
  static constexpr int kThreads = 32 * W;
  static constexpr int kStages = 3;
  static constexpr int kCtas = R == 16 ? 8 / W : W == 8 ? 1 : 12 / W;
  static constexpr int kTile = W * kStep;   // tokens: a step of every warp
  static constexpr int kPart = 3;           // what a part costs beside its own tiles
  static constexpr size_t kCtl = size_t(W) * kStages * kStageBytes;
};

// A part, tiles x .. end - 1 of block b, from token tok0 of its sequence on: `steps` steps, an even share of them a warp's.
struct Part {
  Block b;
  int x, end, tok0, steps;
  template <int W>
  __device__ __forceinline__ void set(int x1) {
    end = min(x1, b.first + b.tiles);
    tok0 = (x - b.first) * (W * kStep);
    steps = (min((end - b.first) * (W * kStep), b.len) - tok0 + kStep - 1) / kStep;
  }
  template <int W>
  __device__ __forceinline__ int first(int warp) const {   // (of warp + 1: behind warp's last)
    return steps * warp / W;
  }
};

template <int R, int W>
struct A4Ctl {
  alignas(128) float4 tokens[W][kStep];                       // of a step's tokens: K's s and z, V's log2 s and z
  LineCtl<W> line;
  Part part[2];                                  // of the sums, by turns (all threads write the same)
  Part ahead[W];                                 // of a warp's copies
  int at[W];                                     // the stage (its bytes in the ring) with the warp's rows at a part's end, or -1
  alignas(8) float m[W][8], l[W][8];             // of eight of the warps' rows, at the end of a part
  uint4 q[R / 8][4][32];                         // the query rows of a part as operands: of eight rows, two k-steps, a lane
  float4 scale[R / 2];                           // of two rows: logits over products, sums of q in their units
  int seen[R];                                   // tokens that the row sees
  Block split[2];                                // parts left for the join
  int last[2];                                   // whether this CTA joins them
};

// How far (log2) a row's largest product passes its reference before that moves. Weights count from 2^(14 - kLazy) there.
constexpr float kLazy = 8.f;

template <int R, int W>
constexpr size_t attend4_smem() {
  return A4Cfg<R, W>::kCtl + sizeof(A4Ctl<R, W>);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 bytes global -> shared (where `here`), zeros where they are not `there` (src is not followed then); a lane's copies so far are a
// group; all but the last N groups have landed.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint64_t policy, uint32_t there) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %3, %2;" ::"r"(dst), "l"(src), "l"(policy), "r"(there)
               : "memory");
}
__device__ __forceinline__ void copy16_if(bool here, uint32_t dst, const void* src, uint64_t policy, uint32_t there) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.s32 p, %4, 0;\n @p cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %3, %2;\n}" ::"r"(dst),
      "l"(src), "l"(policy), "r"(there), "r"(static_cast<int>(here))
      : "memory");
}
__device__ __forceinline__ void copies_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A warp's 8 x 8 matrix of 16-bit elements, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}

// Four of them from shared memory, transposed: lane 8 m + i gives the address of row i of matrix m; register m of lane (g, t) has
// the elements g of the rows 2 t (low) and 2 t + 1.
__device__ __forceinline__ void load_transposed(uint32_t (&d)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
               : "r"(at)
               : "memory");
}

// The 128 bytes around p towards L2 (which all SMs share: what is written there later is seen).
__device__ __forceinline__ void prefetch_line(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// A load that is issued here, not where its value is first needed.
__device__ __forceinline__ uint4 load_now(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
constexpr uint32_t kLargeZ = (127u + 96u) << 23;   // 2^96: sums of up to 2^30 tokens below it stay in fp32
constexpr float kNone = -3e38f;   // a maximum of nothing: finite, so that differences to it are no NaN

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// 2^x down to fp32's last bit (ex2 gives 0 below 2^-126).
__device__ __forceinline__ float ex2_small(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a row's sums are divided by; 0 for a row that saw nothing (its sums are 0).
__device__ __forceinline__ float over(float sum) { return sum == 0.f ? 0.f : rcp(sum); }

__device__ __forceinline__ float low_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

template <int R, int W>
__global__ void __launch_bounds__(A4Cfg<R, W>::kThreads, A4Cfg<R, W>::kCtas)
cache_attend4_kernel(const __grid_constant__ AttendParams P) {
  using C = A4Cfg<R, W>;
  constexpr int kHalves = R / 8;   // pairs of rows of a lane
  constexpr int S = C::kStages;
  extern __shared__ __align__(128) uint8_t smem[];
  static_assert((attend4_smem<R, W>() + 1024) * C::kCtas <= 228 * 1024, "CTAs an SM");
  A4Ctl<R, W>& ctl = *reinterpret_cast<A4Ctl<R, W>*>(smem + C::kCtl);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows = P.q_tokens * P.c.group;
  const int blocks = (rows + R - 1) / R;
  // what the first steps wait for, one after the other, is brought into L2 meanwhile: lengths, table and queries, a line a
  // thread of the grid
  {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * C::kThreads + threadIdx.x;
    const int64_t table_lines = (static_cast<int64_t>(P.n_seq) * P.c.max_pages + 31) >> 5;
    const int64_t q_rows = static_cast<int64_t>(P.n_seq) * P.q_tokens * P.c.hq;
    if (id < table_lines) {
      prefetch_line(P.table + id * 32);
    } else if (id - table_lines < 2 * q_rows) {
      const int row = static_cast<int>((id - table_lines) >> 1), tok = row / P.c.hq;
      prefetch_line(P.q + tok * P.q_st + (row - tok * P.c.hq) * P.q_sh + (id - table_lines & 1) * 64);
    }
  }
  wait_previous_kernel();
  Cuts<C::kPart> cuts;
  line_share<W>(P, blocks, C::kTile, ctl.line, cuts);
  const int x0 = ctl.line.ends[0], x1 = ctl.line.ends[1];
  const int shift = P.c.page_shift;
  const int g = lane >> 2, t = lane & 3;
  // row / group, for groups that are no power of two as for those that are
  const auto row_token = [&](int row) {
    return P.group_inverse ? static_cast<int>(__umulhi(static_cast<uint32_t>(row), P.group_inverse)) : row;
  };
  int splits = 0, now = 0;
  uint8_t* const ring = smem + warp * (S * kStageBytes);
  // K: 16 bytes (t) of the tokens 8 i + g; V: row lane % 8, 16 bytes lane / 8 of eight tokens. A 16-byte chunk c of token r lies
  // at c ^ (r >> 1 & 3): neither meets on a bank
  const auto lies = [](int token, int chunk) { return token * kRowBytes + ((chunk ^ token >> 1) << 4); };
  const uint32_t kget = lies(g, t), vget = lies(lane & 7, lane >> 3);

  // -------------------------------------------------------------- copies, S - 1 steps ahead
  Part& ahead = ctl.ahead[warp];
  const int page_mask = P.c.page - 1;
  const uint32_t page_rows = P.c.heads << shift;
  int held = 0;                       // 32 entries of the sequence's table, a lane each
  int rel = 0, rel_until = INT_MIN;   // the next step's first token in those pages; the end of them or of the warp's steps
  int ahead_pos = 0, ahead_last = 0;  // the part's tokens that those pages begin at, and that the warp's steps end at
  int ahead_head = 0;                 // the head's first row in a page
  const uint32_t ring0 = smem_u32(ring), ring1 = ring0 + S * kStageBytes;
  uint32_t fill = ring0, slot = ring0;   // the stages of the next copies and of the next step
  uint32_t gaps = 0, lost = 0;        // two bits a step, the next one's lowest: pages outside the pool, of its halves; any
  const auto read_table = [&](int at) {   // from token `at` on (looked at in the next fetch)
    const int window = at >> shift;
    ahead_pos = window << shift;
    rel = at - ahead_pos;
    // (the first step that asks for an entry behind those: its second half may be on the next page)
    rel_until = min(ahead_last - ahead_pos, (32 << shift) - 16);
    held = 0;                         // (behind the sequence: nobody sees what is there)
    if (window + lane < (ahead.b.len + page_mask) >> shift)
      held = __ldg(P.table + static_cast<int64_t>(ahead.b.r) * P.c.max_pages + window + lane);
  };
  const auto enter = [&]() {
    const int at = ahead.tok0 + ahead.template first<W>(warp) * kStep;
    ahead_last = ahead.tok0 + ahead.template first<W>(warp + 1) * kStep;
    ahead_head = ahead.b.h << shift;
    ahead_pos = at;
    rel = rel_until = 0;
    if (at < ahead_last) read_table(at);
  };
  const auto settle = [&]() {   // on to a part with something to read
    while (ahead_pos + rel >= ahead_last) {
      Part a = ahead;
      a.x = a.end;
      if (a.x >= x1) {   // no more: pages that are not there
        rel_until = INT_MAX;
        held = -1;
        return;
      }
      next_block(P, blocks, C::kTile, a.b);
      a.template set<W>(x1);
      __syncwarp();
      ahead = a;
      __syncwarp();
      enter();
    }
  };
  // Pages of a call that reads more than L2 keeps leave it first.
  const uint64_t policy = x1 - x0 > 8 ? l2_policy_evict_first() : l2_policy_evict_normal();
  const uint32_t put = lies(g, t);   // eight tokens of K or V at once, 16 bytes a lane
  const uint8_t* const k_base = P.c.k + lane * 16;
  const uint8_t* const v_base = P.c.v + lane * 16;
  // the rows' numbers: four lanes each for the halves of K's and of V's
  const uint32_t* const numbers = (lane & 8 ? P.c.v_param : P.c.k_param) + (lane & 3) * 4;
  // The copies of the next step, in three pieces that stand between the products: where its rows are (of its two halves, in
  // the pool), K, and the rest.
  uint32_t row0 = 0, row1 = 0;
  uint32_t ok0 = 0, ok1 = 0;   // bytes of each copy: 16, or 0 for a page outside the pool (or no step)
  const auto find = [&]() {
    const int id0 = __shfl_sync(0xffffffffu, held, rel >> shift);
    const int id1 = __shfl_sync(0xffffffffu, held, (rel + 16) >> shift);
    ok0 = static_cast<uint32_t>(id0) < static_cast<uint32_t>(P.c.num_pages) ? 16 : 0;
    ok1 = static_cast<uint32_t>(id1) < static_cast<uint32_t>(P.c.num_pages) ? 16 : 0;
    gaps = gaps >> 2 | (ok0 ^ 16) << 2 * (S - 3) | (ok1 ^ 16) << (2 * (S - 3) + 1);   // (bits 2 (S - 1) and the next)
    row0 = static_cast<uint32_t>(id0) * page_rows + ahead_head + (rel & page_mask);
    row1 = static_cast<uint32_t>(id1) * page_rows + ahead_head + (rel + 16 & page_mask);
  };
  const auto copy_codes = [&](const uint8_t* base, uint32_t to) {
    const uint8_t* const from0 = base + static_cast<uint64_t>(row0) * kRowBytes;
    const uint8_t* const from1 = base + static_cast<uint64_t>(row1) * kRowBytes;
    copy16(to, from0, policy, ok0);
    copy16(to + 512, from0 + 512, policy, ok0);
    copy16(to + 1024, from1, policy, ok1);
    copy16(to + 1536, from1 + 512, policy, ok1);
  };
  const auto copy_keys = [&]() { copy_codes(k_base, fill + put); };
  const auto copy_rest = [&]() {
    copy_codes(v_base, fill + put + kCodeBytes);
    copy16_if(lane < 16, fill + kNumbers + lane * 16, numbers + (lane & 4 ? row1 : row0), policy, lane & 4 ? ok1 : ok0);
    copies_group();   // (an empty one too: groups are counted)
    fill += kStageBytes;
    if (fill == ring1) fill = ring0;
    rel += kStep;
    if (rel >= rel_until) {
      if (ahead_pos + rel < ahead_last)
        read_table(ahead_pos + rel);
      else
        settle();
    }
  };
  // the raw query rows of a part: row 8 e + g of the block, elements 32 t .. 32 t + 31
  uint4 raw[kHalves][4];
  const auto load_rows = [&](const Block& b) {
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      const int row = b.rb * R + 8 * e + g;
      const int qt = row_token(row), hq = b.h * P.c.group + row - qt * P.c.group;
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[e][i] = make_uint4(0, 0, 0, 0);
      if (row < rows) {
        const uint16_t* from = P.q + (static_cast<int64_t>(b.r) * P.q_tokens + qt) * P.q_st + hq * P.q_sh + 32 * t;
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[e][i] = load_now(from + 8 * i);
      }
    }
  };
  // A part's query rows as operands, in shared memory: every warp has them in `raw` and looks for their largest magnitudes; the
  // conversion is dealt to the warps. (In registers they would be 32 of a thread's with 16 rows, and converted by all.)
  const auto convert = [&](const Block& b) {
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      const uint32_t* u = &raw[e][0].x;
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
      if (warp == W - 1 && t == 0) {
        float* const to = reinterpret_cast<float*>(&ctl.scale[(8 * e + g) / 2]) + (g & 1);
        to[0] = P.alpha * __uint_as_float(static_cast<uint32_t>(min(24 - up, 127) + 127) << 23);
        to[2] = ex >= 127 + 112 ? __uint_as_float(0x7fc00000u) : sum * scale * 5.9604644775390625e-8f;   // 2^-24
        const int row = b.rb * R + 8 * e + g;
        ctl.seen[8 * e + g] = row < rows ? b.len - P.q_tokens + row_token(row) + 1 : 0;
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {   // 8 elements: n and n + 4 go together
        if (w % W != warp) continue;
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[2 * i] = low_bf16(u[4 * w + i]) * scale;
          f[2 * i + 1] = high_bf16(u[4 * w + i]) * scale;
        }
        ctl.q[e][w][lane] = make_uint4(f16x2(f[0], f[4]), f16x2(f[1] * 0.0625f, f[5] * 0.0625f), f16x2(f[2], f[6]),
                                       f16x2(f[3] * 0.0625f, f[7] * 0.0625f));
      }
    }
  };
  if (x0 < x1) {
    Part a;
    a.b = ctl.line.first;
    a.x = x0;
    a.template set<W>(x1);
    ctl.part[0] = ahead = a;
    __syncwarp();
    enter();
    load_rows(a.b);
    settle();
    find();
    copy_keys();
    copy_rest();
    convert(a.b);
    __syncthreads();
  }
  for (int x = x0; x < x1;) {
    const Part& part = ctl.part[now];
    const Block& b = part.b;
    if (x == x0) {   // (not before: the queries' exchanges would wait behind these copies)
#pragma unroll 1
      for (int i = 1; i < S - 1; ++i) {
        find();
        copy_keys();
        copy_rest();
      }
    }

    // ---------------------------------------------------------- the steps
    // this lane's rows are 8 e + 2 t and 8 e + 2 t + 1, its tokens 8 i + g
    float o[8][kHalves][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < kHalves; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][e][k] = 0.f;
    float2 m[kHalves], top[kHalves], l[kHalves], z[kHalves];   // the lane's maxima; the rows' references; the lane's sums of p, p z
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      m[e] = top[e] = both(kNone);
      l[e] = z[e] = both(0.f);
    }
    float unit = 1.f;   // of z
    const int first = part.template first<W>(warp), last = part.template first<W>(warp + 1);
    const int tok0 = part.tok0, all_see = b.len - P.q_tokens + 1;
#pragma unroll 1
    for (int step = first; step < last; ++step) {
      copies_wait<S - 2>();
      __syncwarp();   // every lane's copies of this step have landed, and the step before has been read
      find();
      copy_keys();
      const uint8_t* const at = ring + (slot - ring0);
      {
        // a lane a token: its four numbers for every lane
        const uint32_t* const n = reinterpret_cast<const uint32_t*>(at + kNumbers);
        const uint32_t a = n[lane], c = n[kStep + lane];
        if (__any_sync(0xffffffffu, (c & 0x7f800000u) >= kLargeZ) && unit == 1.f) {   // (as the sum so far)
          unit = ex2(-len_bits(b.len));
#pragma unroll
          for (int e = 0; e < kHalves; ++e) z[e] = fmul2(z[e], both(unit));
        }
        ctl.tokens[warp][lane] = make_float4(low_bf16(a), high_bf16(a), lg2(low_bf16(c)), high_bf16(c) * unit);
      }
      float s[2][kHalves][4];
      {
        uint4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const uint4*>(at + i * (8 * kRowBytes) + kget);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < kHalves; ++e)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[k][e][r] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint4 q[kHalves];
#pragma unroll
          for (int e = 0; e < kHalves; ++e) q[e] = ctl.q[e][w][lane];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k) {   // (the two halves' products one between the other: each waits for its own)
              const uint32_t ua = h ? (&u[2 * k].x)[w] >> 8 : (&u[2 * k].x)[w];
              const uint32_t ub = h ? (&u[2 * k + 1].x)[w] >> 8 : (&u[2 * k + 1].x)[w];
              const uint32_t a[4] = {ua & 0x000f000fu, ub & 0x000f000fu, ua & 0x00f000f0u, ub & 0x00f000f0u};
#pragma unroll
              for (int e = 0; e < kHalves; ++e) mma_f16(s[k][e], a, h ? q[e].z : q[e].x, h ? q[e].w : q[e].y);
            }
        }
      }
      copy_rest();
      __syncwarp();
      const int pos0 = tok0 + step * kStep;
      const uint32_t hole = gaps & 3u;
      lost |= hole;
      const bool some = hole != 0 || pos0 + kStep > all_see;   // tokens that not all rows see
      // logits (over kq) in place of the products
      float2 y[4][kHalves], kq[kHalves];
      float ls[4];
#pragma unroll
      for (int e = 0; e < kHalves; ++e) {
        const float4 c = ctl.scale[4 * e + t];
        kq[e] = make_float2(c.x, c.y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 f = ctl.tokens[warp][8 * i + g];
          ls[i] = f.z;
          y[i][e] = ffma2(both(f.x), make_float2(s[i / 2][e][2 * (i & 1)], s[i / 2][e][2 * (i & 1) + 1]),
                          fmul2(both(f.y), make_float2(c.z, c.w)));
        }
      }
      if (some) {
#pragma unroll
        for (int e = 0; e < kHalves; ++e) {
          const int s0 = ctl.seen[8 * e + 2 * t], s1 = ctl.seen[8 * e + 2 * t + 1];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int pos = pos0 + 8 * i + g;
            const bool gone = hole >> (i >> 1) & 1u;
            if (gone || pos >= s0) y[i][e].x = -INFINITY;
            if (gone || pos >= s1) y[i][e].y = -INFINITY;
          }
        }
      }
      // the lane's own largest logits, and the rows' references of the products within 2^kLazy of the largest so far
      float2 tx[kHalves];
      bool moved = false;
#pragma unroll
      for (int e = 0; e < kHalves; ++e) {
        float2 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = ffma2(y[i][e], kq[e], both(ls[i]));
        tx[e] = make_float2(max3(fmaxf(w[0].x, w[1].x), w[2].x, w[3].x), max3(fmaxf(w[0].y, w[1].y), w[2].y, w[3].y));
        float2 mx = make_float2(max3(fmaxf(y[0][e].x, y[1][e].x), y[2][e].x, y[3][e].x),
                                max3(fmaxf(y[0][e].y, y[1][e].y), y[2][e].y, y[3][e].y));
        mx = fmul2(mx, kq[e]);
        mx = make_float2(fmaxf(mx.x, m[e].x), fmaxf(mx.y, m[e].y));
        const float2 kept = make_float2(ex2(m[e].x - mx.x), ex2(m[e].y - mx.y));
        m[e] = mx;
        l[e] = fmul2(l[e], kept);
        z[e] = fmul2(z[e], kept);
        moved |= tx[e].x > top[e].x + kLazy || tx[e].y > top[e].y + kLazy;
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int e = 0; e < kHalves; ++e) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) {
            tx[e].x = fmaxf(tx[e].x, __shfl_xor_sync(0xffffffffu, tx[e].x, d));
            tx[e].y = fmaxf(tx[e].y, __shfl_xor_sync(0xffffffffu, tx[e].y, d));
          }
          tx[e] = make_float2(fmaxf(tx[e].x, top[e].x), fmaxf(tx[e].y, top[e].y));
          const float f0 = ex2(top[e].x - tx[e].x), f1 = ex2(top[e].y - tx[e].y);
          top[e] = tx[e];
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
          const float2 mr = make_float2(-m[e].x, -m[e].y);
          const float2 tr = make_float2(14.f - kLazy - top[e].x, 14.f - kLazy - top[e].y);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float vz = ctl.tokens[warp][8 * i + g].w;
            const float2 a = ffma2(y[i][e], kq[e], mr);
            const float2 p = make_float2(ex2(a.x), ex2(a.y));
            const float2 c = fadd2(ffma2(y[i][e], kq[e], both(ls[i])), tr);
            float2 ww = make_float2(ex2(c.x), ex2(c.y)), zz = both(vz);
            if constexpr (kSome.value) {
              // (a NaN of a token that the row does not see stays out: some rows of the step may see it)
              if (y[i][e].x == -INFINITY) ww.x = zz.x = 0.f;
              if (y[i][e].y == -INFINITY) ww.y = zz.y = 0.f;
            }
            l[e] = fadd2(l[e], p);
            z[e] = ffma2(p, zz, z[e]);
            w[i][e] = f16x2(ww.x, ww.y);
          }
        }
      };
      if (some)
        weigh(std::true_type{});
      else
        weigh(std::false_type{});
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < kHalves; ++e) w[i][e] = transposed(w[i][e]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t c0[4], c1[4];   // four codes of two tokens each
        const uint32_t from = slot + kCodeBytes + 2 * k * (8 * kRowBytes) + vget;
        load_transposed(c0, from);
        load_transposed(c1, from + 8 * kRowBytes);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            // low codes, and low + 16 high ones: the end takes the former's sum out of the latter's
            const uint32_t ua = h ? __byte_perm(c0[i], 0, 0x4341) : c0[i] & 0x00ff00ffu;
            const uint32_t ub = h ? __byte_perm(c1[i], 0, 0x4341) : c1[i] & 0x00ff00ffu;
            const uint32_t a[4] = {ua & 0x000f000fu, ua, ub & 0x000f000fu, ub};
#pragma unroll
            for (int e = 0; e < kHalves; ++e) mma_f16(o[2 * i + h][e], a, w[2 * k][e], w[2 * k + 1][e]);
          }
      }
      slot += kStageBytes;
      if (slot == ring1) slot = ring0;
    }

    // ---------------------------------------------------------- the end of a part: the warps' rows together, eight by eight
    const bool has = first < last, whole = x == b.first && part.end == b.first + b.tiles;
    float* const out = P.partial + (static_cast<int64_t>(blockIdx.x) * 2 + (x == b.first)) * kAttend4PartWords;
    // (in the stage of the last step, which the next one's copies will fill)
    const int stage = (slot == ring0 ? ring1 : slot) - kStageBytes - ring0;
    float* const mine = reinterpret_cast<float*>(ring + stage);
    if (lane == 0) ctl.at[warp] = has ? stage : -1;
    const int next_x = part.end;
#pragma unroll
    for (int e = 0; e < kHalves; ++e) {
      if (has) {
        float2 all = m[e];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          all.x = fmaxf(all.x, __shfl_xor_sync(0xffffffffu, all.x, d));
          all.y = fmaxf(all.y, __shfl_xor_sync(0xffffffffu, all.y, d));
        }
        const float2 kept = make_float2(ex2(m[e].x - all.x), ex2(m[e].y - all.y));
        float2 ll = fmul2(l[e], kept), zz = fmul2(z[e], kept);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          ll.x += __shfl_xor_sync(0xffffffffu, ll.x, d);
          ll.y += __shfl_xor_sync(0xffffffffu, ll.y, d);
          zz.x += __shfl_xor_sync(0xffffffffu, zz.x, d);
          zz.y += __shfl_xor_sync(0xffffffffu, zz.y, d);
        }
        // The warp's averages, as quarters, so that neither sum p s c nor sum p z alone passes the largest float: products of c 2^-24
        // or 16 c 2^-24 with weights times 2^(14 - kLazy). Averages keep the bits of values near either end of fp32, which sums of
        // fractions of them would lose.
        const float ov[2] = {over(ll.x), over(ll.y)}, back = 0.25f / unit;
        const float f[2] = {ex2_small(top[e].x - all.x), ex2_small(top[e].y - all.y)};
        const float zq[2] = {zz.x * ov[0] * back, zz.y * ov[1] * back};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float4 v;
            v.x = fmaf(o[2 * i][e][j] * (65536.f * ov[j]), f[j], zq[j]);
            v.y = fmaf((o[2 * i][e][2 + j] - o[2 * i][e][j]) * (4096.f * ov[j]), f[j], zq[j]);
            v.z = fmaf(o[2 * i + 1][e][j] * (65536.f * ov[j]), f[j], zq[j]);
            v.w = fmaf((o[2 * i + 1][e][2 + j] - o[2 * i + 1][e][j]) * (4096.f * ov[j]), f[j], zq[j]);
            // columns 32 i + 4 g of row 2 t + j; 16 bytes c of row r lie at c ^ (r & 6)
            reinterpret_cast<float4*>(mine + (2 * t + j) * kHeadDim)[(8 * i + g) ^ (2 * t)] = v;
          }
        if (g == 0) {
          *reinterpret_cast<float2*>(&ctl.m[warp][2 * t]) = all;
          *reinterpret_cast<float2*>(&ctl.l[warp][2 * t]) = ll;
        }
      }
      if (e + 1 == kHalves && next_x < x1) {   // the next part, and its rows on their way
        Part a = part;
        a.x = next_x;
        next_block(P, blocks, C::kTile, a.b);
        a.template set<W>(x1);
        load_rows(a.b);
        ctl.part[now ^ 1] = a;
        __syncwarp();
      }
      __syncthreads();
      for (int row = warp; row < 8; row += W) {
        float f[W], mx = kNone, sum = 0.f;
        float4 v[W], a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) {   // (a warp without steps has nothing there)
          const int at = ctl.at[w];
          f[w] = at >= 0 ? ctl.m[w][row] : kNone;
          v[w] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (at >= 0)
            v[w] = reinterpret_cast<const float4*>(smem + w * (S * kStageBytes) + at + row * (kHeadDim * 4))[lane ^ (row & 6)];
          mx = fmaxf(mx, f[w]);
        }
#pragma unroll
        for (int w = 0; w < W; ++w) {   // (shares of the sum)
          f[w] = ctl.at[w] >= 0 ? ctl.l[w][row] * ex2(f[w] - mx) : 0.f;
          sum += f[w];
        }
        const float ov = over(sum);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          f[w] *= ov;
          a.x = fmaf(v[w].x, f[w], a.x);
          a.y = fmaf(v[w].y, f[w], a.y);
          a.z = fmaf(v[w].z, f[w], a.z);
          a.w = fmaf(v[w].w, f[w], a.w);
        }
        const int r = 8 * e + row;
        if (whole) {
          emit_row(P, b, b.rb * R + r, rows, row_token, a, mx, sum, lane);
        } else {
          reinterpret_cast<float4*>(out + r * kHeadDim)[lane] = a;
          if (lane == 0) {
            out[R * kHeadDim + r] = mx;
            out[R * kHeadDim + R + r] = sum;
          }
        }
      }
      if (!whole && e == 0) {
        if (threadIdx.x == 0) ctl.split[splits] = b;
        ++splits;
      }
      if (e + 1 == kHalves && next_x < x1) convert(ctl.part[now ^ 1].b);   // (no warp needs this part's rows any more)
      __syncthreads();   // the sums have been read
    }
    x = next_x;
    now ^= 1;
  }

  copies_wait<0>();   // (the empty ones behind the last step write zeros into the ring)
  if (lost && lane == 0) atomicOr(P.err, kErrCheck);

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
  __syncthreads();   // every thread's part of the sums is out, and ctl.split is written
  if (threadIdx.x < splits) {
    int w0, w1;
    cuts.parts(ctl.split[threadIdx.x], &w0, &w1);
    ctl.last[threadIdx.x] = inc_acq_rel_gpu(P.arrive + w0, static_cast<unsigned>(w1 - w0)) == static_cast<unsigned>(w1 - w0);
  }
  __syncthreads();
  constexpr int kRows = (R + W - 1) / W;
  for (int n = 0; n < splits; ++n) {
    if (!ctl.last[n]) continue;
    const Block s = ctl.split[n];
    int w0, w1;
    cuts.parts(s, &w0, &w1);
    // A warp has the rows warp, warp + W, ...; where there are twice as many warps as rows or more, a row's parts are dealt
    // to several warps, whose sums the first of them adds in their order.
    const int parts = w1 - w0 + 1, there = min(R, rows - s.rb * R);
    const int teams = kRows == 1 && there < W ? W / there : 1;
    const int row0 = teams > 1 ? warp % there : warp, team = teams > 1 ? warp / there : 0;
    const int p0 = parts * team / teams, p1 = parts * (team + 1) / teams;
    const bool works = row0 < there && team < teams;
    // part p: slot 0 of CTA w0 + p, of the first one slot 1
    const auto at = [&](int p) { return P.partial + (static_cast<int64_t>(w0 + p) * 2 + (p == 0)) * kAttend4PartWords; };
    float mx[kRows], sum[kRows];
    float4 acc[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      mx[k] = kNone;
      sum[k] = 0.f;
      acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    constexpr int kAtOnce = kRows == 1 ? 20 : 16 / kRows;   // parts of each row whose loads are in flight
    for (int c0 = p0; works && c0 < p1; c0 += 32) {
      const int count = min(p1 - c0, 32);
      float4 v[kAtOnce][kRows];
      const auto load = [&](int j0) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            v[j][k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (j0 + j < count && row0 + k * W < there)
              v[j][k] = __ldcg(reinterpret_cast<const float4*>(at(c0 + j0 + j) + (row0 + k * W) * kHeadDim) + lane);
          }
      };
      float pm[kRows], pl[kRows];   // a lane a part: its maximum and sum
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int row = row0 + k * W;
        pm[k] = kNone;
        pl[k] = 0.f;
        if (lane < count && row < there) {
          pm[k] = __ldcg(at(c0 + lane) + R * kHeadDim + row);
          pl[k] = __ldcg(at(c0 + lane) + R * kHeadDim + R + row);
        }
      }
      load(0);
      float f[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const float top = fmaxf(mx[k], warp_max(pm[k])), kept = sum[k] * ex2(mx[k] - top);
        mx[k] = top;
        pl[k] *= ex2(pm[k] - top);
        f[k] = pl[k];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) pl[k] += __shfl_xor_sync(0xffffffffu, pl[k], d);
        sum[k] = kept + pl[k];
        const float ov = over(sum[k]), back = kept * ov;
        f[k] *= ov;
        acc[k].x *= back, acc[k].y *= back, acc[k].z *= back, acc[k].w *= back;
      }
      for (int j0 = 0;;) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            const float g = __shfl_sync(0xffffffffu, f[k], (j0 + j) & 31);
            if (j0 + j >= count) continue;
            acc[k].x = fmaf(v[j][k].x, g, acc[k].x);
            acc[k].y = fmaf(v[j][k].y, g, acc[k].y);
            acc[k].z = fmaf(v[j][k].z, g, acc[k].z);
            acc[k].w = fmaf(v[j][k].w, g, acc[k].w);
          }
        j0 += kAtOnce;
        if (j0 >= count) break;
        load(j0);
      }
    }
    if (teams > 1) {
      float4* const sums = reinterpret_cast<float4*>(smem);
      __syncthreads();   // (the block before has read its sums)
      if (works) sums[warp * 32 + lane] = acc[0];
      if (works && lane == 0) {
        ctl.m[warp][0] = mx[0];
        ctl.l[warp][0] = sum[0];
      }
      __syncthreads();
      if (works && team == 0)
        for (int w = row0 + there; w < teams * there; w += there) {
          const float top = fmaxf(mx[0], ctl.m[w][0]);
          const float mine = sum[0] * ex2(mx[0] - top), other = ctl.l[w][0] * ex2(ctl.m[w][0] - top);
          const float4 v = sums[w * 32 + lane];
          mx[0] = top;
          sum[0] = mine + other;
          const float ov = over(sum[0]), a = mine * ov, c = other * ov;
          acc[0] = make_float4(fmaf(acc[0].x, a, v.x * c), fmaf(acc[0].y, a, v.y * c), fmaf(acc[0].z, a, v.z * c),
                               fmaf(acc[0].w, a, v.w * c));
        }
    }
    if (works && team == 0)
#pragma unroll
      for (int k = 0; k < kRows; ++k)
        if (row0 + k * W < there)
          emit_row(P, s, s.rb * R + row0 + k * W, rows, row_token, acc[k], mx[k], sum[k], lane);
  }
}

template <int R, int W>
cudaError_t attend4_rows(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  using C = A4Cfg<R, W>;
  constexpr size_t smem = attend4_smem<R, W>();
  static_assert(C::kCtas <= kAttend4Ctas, "parts in the workspace");
  auto* fn = cache_attend4_kernel<R, W>;
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  // no more CTAs than there can be tiles
  const int64_t blocks = (p.q_tokens * p.c.group + R - 1) / R;
  const int64_t tiles = ((static_cast<int64_t>(p.c.max_pages) << p.c.page_shift) + C::kTile - 1) / C::kTile;
  const int64_t most = static_cast<int64_t>(C::kCtas) * c.sms;
  const int64_t want = tiles >= most ? most : tiles * p.n_seq * p.c.heads * blocks;
  return launch_after_previous(fn, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(C::kThreads), smem, stream, p);
}

template <int W>
cudaError_t attend4_warps(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  return p.q_tokens * p.c.group > 8 ? attend4_rows<16, W>(c, p, stream) : attend4_rows<8, W>(c, p, stream);
}

}  // namespace

cudaError_t launch_cache4_attend(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  const int64_t rows = static_cast<int64_t>(p.q_tokens) * p.c.group;
  const int64_t blocks = static_cast<int64_t>(p.n_seq) * p.c.heads * (rows > 8 ? (rows + 15) / 16 : 1);
  const int64_t longest = static_cast<int64_t>(p.c.max_pages) << p.c.page_shift;
  // Few warps a CTA make the end of a part cheap, many cut a block into fewer parts and its steps among more. (Figures of both sides from
  // the same day, with tables as wide as the longest sequence; today's are up to 2% more.)
  // Three blocks an SM or more: 2 warps a CTA. (8 heads; 2 against 4 warps: 64 ragged sequences 46.2 and 46.9 us, 400 of 100 to 8000
  // tokens 129 and 136, 400 of 20 to 800 34.7 and 41.7, 1000 of 64 42.2 and 63.3; 50 of 200 to 800, 400 blocks, 15.8 and 13.0. 16
  // rows: 100 of 100 to 3000 39.5 and 41.9, 400 of 20 to 800 64 and 78.)
  if (blocks >= 3 * c.sms) return attend4_warps<2>(c, p, stream);
  // No more than one block an SM and a table that holds short ones only (lengths are not known here, so a wider table takes 4 warps for
  // short ones too: 16 of 96 to 700 with a table of 16384 tokens 7.7 for 6.6): 8 warps. (8 against 4: 16 of 96 to 700 6.6 and 7.6, 8 of 100 to
  // 800 7.4 and 8.1, 8 of 500 to 2000 11.5 and 12.0, 19 of 50 to 1000 8.6 and 10.4; 24, 192 blocks, 10.5 and 8.8, 4 of 200 to 3000
  // 13.3 and 11.0, 8 of 32768 56.3 and 51.0, one of 131072 32.0 and 32.8. 16 rows: 16 of 100 to 700 12.1 and 12.6, 19 of 100 to 2000
  // 16.4 and 17.4.)
  if (blocks <= c.sms && longest <= 2048) return attend4_warps<8>(c, p, stream);
  return attend4_warps<4>(c, p, stream);
}

}  // namespace kve
