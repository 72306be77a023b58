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
//   p = hi + mid / 16 + lo / 256, three pieces: a relative 2^-12, below 2^-4 of the final bf16 rounding.
//     Two pieces would be the 2^-8 that bf16 probabilities have.
// Statistics, sums and the output accumulate in fp32 registers: a tile's O^T is added to them scaled by
// exp(old maximum - new), so TMEM holds one tile's products and is never rescaled.
//
// The work is cut over the tokens: all (sequence, head, row block)s' tiles in one line, an equal share of it
// for each of two CTAs an SM, whatever the lengths (the lengths are read on the GPU: a captured call serves
// every later length). A block that falls to several CTAs is joined by the one that finishes last, from
// their fp32 parts in token order, so the sum does not depend on who that is.
#include "kve_internal.h"
#include "kve_ptx.cuh"

namespace kve {
namespace {

constexpr int kAttendThreads = 192;   // 4 softmax warps, TMA producer, MMA issuer
constexpr int kStages = 3;            // K and V tiles in flight: 96 KB a CTA, 192 KB an SM
constexpr int kTileBytes = kTileKeys * kHeadDim;
constexpr int kMostTilePages = kTileKeys / 16;

constexpr int up16(int x) { return (x + 15) / 16 * 16; }

template <int R>
struct ACfg {
  static constexpr int kNs = up16(2 * R);           // columns of S^T: q's hi rows, then its lo rows
  static constexpr int kNp = up16(3 * R);           // columns of O^T: p's hi, mid and lo rows
  static constexpr int kOCol = kNs;
  static constexpr int kTmemCols = kNs + kNp <= 32 ? 32 : kNs + kNp <= 64 ? 64 : 128;
  static constexpr uint32_t kIdescS = idesc_e4m3_f32(128, kNs, false);
  static constexpr uint32_t kIdescO = idesc_e4m3_f32(128, kNp, true);
  static constexpr size_t kQ = size_t(kStages) * 2 * kTileBytes;
  static constexpr size_t kP = kQ + kNs * kHeadDim;
  static constexpr size_t kCtl = kP + kNp * kTileKeys;
};

template <int R>
struct ACtl {
  uint64_t full[kStages], empty[kStages];
  uint64_t s_full, p_full, o_full, q_full, meet, drain;
  float ks[kStages][kMostTilePages], vs[kStages][kMostTilePages];
  uint32_t pages[kStages];          // bit j: page j of the tile holds tokens
  float red[2][4][R];               // row maxima of the warps, by tile parity (and row sums of a part)
  float qs[2][R];                   // log2(e) / sqrt(d) / the power of two in the q pieces, by part parity
  unsigned long long sums[kAttendThreads / 32];
  long long base;                   // tiles in front of the first part's sequence
  int first_r, last;
  uint32_t tmem_base;
  int abort, never;   // never: stays 0 (waits that a given-up call still has to make)
};

template <int R>
constexpr size_t attend_smem() {
  return ACfg<R>::kCtl + sizeof(ACtl<R>) + 1024;   // the tiles start on 1024 bytes
}

// Walks a CTA's share of the line of tiles, part by part: (sequence, head, row block)s in this order.
struct Walk {
  int r, h, rb, tiles, len;
  long long first;   // the block's first tile in the line

  __device__ __forceinline__ static int length(const AttendParams& P, int r) {
    const int len = __ldg(P.lens + r);
    return min(max(len, 0), P.c.max_pages << P.c.page_shift);
  }
  __device__ __forceinline__ void enter(const AttendParams& P, int seq) {
    r = seq;
    len = length(P, r);
    tiles = (len + kTileKeys - 1) / kTileKeys;
  }
  // The block that holds tile x, for x at or behind the first tile of sequence seq (base).
  __device__ __forceinline__ void seek(const AttendParams& P, int blocks, int seq, long long base, long long x) {
    enter(P, seq);
    const long long at = (x - base) / tiles;
    h = static_cast<int>(at / blocks);
    rb = static_cast<int>(at - static_cast<long long>(h) * blocks);
    first = base + at * tiles;
  }
  __device__ __forceinline__ void next(const AttendParams& P, int blocks) {
    first += tiles;
    if (++rb < blocks) return;
    rb = 0;
    if (++h < P.c.heads) return;
    h = 0;
    do enter(P, r + 1);
    while (tiles == 0);   // a tile follows, so a sequence that is not empty does
  }
};

// The power of two that brings the largest magnitude (bf16 bits a, finite) into [128, 256), as fp32 bits.
__device__ __forceinline__ uint32_t piece_scale(uint32_t a) {
  const int e = 261 - static_cast<int>(a >> 7);   // 2^(7 - (x - 127)), biased
  return static_cast<uint32_t>(min(e, 253)) << 23;
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ float2 e4m3x2_values(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  float2 f;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}

__device__ __forceinline__ uint16_t to_bf16(float x) {
  uint16_t d;
  asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(d) : "f"(x));
  return d;
}

template <int R>
__global__ void __launch_bounds__(kAttendThreads, kAttendCtas)
cache_attend_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ AttendParams P) {
  using C = ACfg<R>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  ACtl<R>& ctl = *reinterpret_cast<ACtl<R>*>(smem + C::kCtl);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rows = P.q_tokens * P.c.group;
  const int blocks = (rows + R - 1) / R;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&ctl.full[i], 2);    // the bytes, and the scales beside them
      mbar_init(&ctl.empty[i], 1);
    }
    mbar_init(&ctl.s_full, 1);
    mbar_init(&ctl.p_full, 4);
    mbar_init(&ctl.o_full, 1);
    mbar_init(&ctl.q_full, 4);
    mbar_init(&ctl.meet, 4);
    mbar_init(&ctl.drain, 1);
    ctl.abort = ctl.never = 0;
    fence_mbar_init();
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  wait_previous_kernel();
  if (warp == 5) {
    tmem_alloc(&ctl.tmem_base, C::kTmemCols);
    tmem_relinquish();
  }
  // The line's length, and the sequence in which this CTA's share starts: a run of sequences a thread
  const int cap = P.c.max_pages << P.c.page_shift;
  const int per = (P.n_seq + kAttendThreads - 1) / kAttendThreads;
  const int s0 = min(tid * per, P.n_seq), s1 = min(s0 + per, P.n_seq);
  long long mine = 0;
  bool bad = false;
  for (int r = s0; r < s1; ++r) {
    const int len = __ldg(P.lens + r);
    bad |= len < 0 || len > cap;
    mine += (min(max(len, 0), cap) + kTileKeys - 1) / kTileKeys;
  }
  if (bad && blockIdx.x == 0) atomicOr(P.err, kErrCheck);
  const long long own = mine * (static_cast<long long>(P.c.heads) * blocks);
  long long front = own;   // tiles up to and with this thread's sequences
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, front, o);
    if (lane >= o) front += x;
  }
  if (lane == 31) ctl.sums[warp] = static_cast<unsigned long long>(front);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < kAttendThreads / 32; ++w) {
    if (w < warp) front += static_cast<long long>(ctl.sums[w]);
    total += static_cast<long long>(ctl.sums[w]);
  }
  front -= own;
  const int ctas = static_cast<int>(min(total, static_cast<long long>(gridDim.x)));   // those that have a share
  const bool works = static_cast<int>(blockIdx.x) < ctas;
  const auto share = [&](long long w) { return total * w / ctas; };                    // first tile of CTA w
  const long long x0 = works ? share(blockIdx.x) : 0, x1 = works ? share(blockIdx.x + 1) : 0;
  if (works && own > 0 && x0 >= front && x0 < front + own) {
    long long at = front;
    for (int r = s0; r < s1; ++r) {
      const long long n = (Walk::length(P, r) + kTileKeys - 1) / kTileKeys * (static_cast<long long>(P.c.heads) * blocks);
      if (x0 < at + n) {
        ctl.first_r = r;
        ctl.base = at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  const uint32_t tmem = ctl.tmem_base;
  const auto fail = [&]() {
    ctl.abort = 1;
    atomicOr(P.err, kErrWait);
  };

  if (warp == 4) {
    // ------------------------------------------------------------ producer: lane j the tile's page j
    if (works) {
      const int tile_pages = kTileKeys >> P.c.page_shift, page_bytes = P.c.page * kHeadDim;
      Walk at;
      at.seek(P, blocks, ctl.first_r, ctl.base, x0);
      long long x = x0;
      // the page of this lane in tile x (-1: none), and its scales
      const auto page_of = [&](const Walk& w, long long tile) {
        const int j = static_cast<int>(tile - w.first) * tile_pages + lane;
        const bool has = lane < tile_pages && (j << P.c.page_shift) < w.len;
        return has ? __ldg(P.table + static_cast<int64_t>(w.r) * P.c.max_pages + j) : -1;
      };
      const auto valid = [&](int id) { return id >= 0 && id < P.c.num_pages; };
      int id = page_of(at, x);
      bool more = true;
      int it = 0;
      for (; more; ++it) {
        const int st = it % kStages;
        const bool has = lane < tile_pages && ((static_cast<int>(x - at.first) * tile_pages + lane) << P.c.page_shift) < at.len;
        const bool ok = valid(id);
        if (has && !ok) atomicOr(P.err, kErrCheck);
        const int64_t block = static_cast<int64_t>(ok ? id : 0) * P.c.heads + at.h;
        float ks = 0.f, vs = 0.f;
        if (ok) {
          ks = __ldg(P.c.k_scale + block);
          vs = __ldg(P.c.v_scale + block);
        }
        // the next tile's page while this one waits
        Walk then = at;
        more = x + 1 < x1;
        if (more && x + 1 == then.first + then.tiles) then.next(P, blocks);
        const int next_id = more ? page_of(then, x + 1) : -1;
        if (!warp_wait(&ctl.empty[st], ((it / kStages) & 1) ^ 1, P.wait_limit_ns, &ctl.abort)) {
          if (lane == 0) fail();
          break;
        }
        const uint32_t mask = __ballot_sync(0xffffffffu, ok);
        if (lane == 0) mbar_arrive_expect_tx(&ctl.full[st], __popc(mask) * 2 * page_bytes);
        __syncwarp();
        if (ok) {
          uint8_t* kdst = smem + static_cast<size_t>(st) * 2 * kTileBytes + lane * page_bytes;
          const int row = static_cast<int>(block << P.c.page_shift);
          tma_load_2d(kdst, &tm_k, 0, row, &ctl.full[st]);
          tma_load_2d(kdst + kTileBytes, &tm_v, 0, row, &ctl.full[st]);
        }
        if (lane < kMostTilePages) {
          ctl.ks[st][lane] = ks;
          ctl.vs[st][lane] = vs;
        }
        if (lane == 0) ctl.pages[st] = mask;
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.full[st]);
        id = next_id;
        at = then;
        ++x;
      }
      // after a wait that ran out: the copies in flight end before the shared memory does
      if (ctl.abort && lane == 0) {
        for (int k = max(it - kStages, 0); k < it; ++k)
          mbar_wait(&ctl.full[k % kStages], (k / kStages) & 1, P.wait_limit_ns, &ctl.never);
      }
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------ MMA issuer
    if (works && lane == 0) {
      const uint32_t kaddr = smem_u32(smem), qaddr = kaddr + static_cast<uint32_t>(C::kQ);
      const uint32_t paddr = kaddr + static_cast<uint32_t>(C::kP);
      Walk at;
      at.seek(P, blocks, ctl.first_r, ctl.base, x0);
      const int n = static_cast<int>(x1 - x0);
      int part = 0;
      long long x = x0;
      const auto scores = [&](int it, bool new_q) -> bool {
        if (new_q && !mbar_wait(&ctl.q_full, part++ & 1, P.wait_limit_ns, &ctl.abort)) return false;
        if (!mbar_wait(&ctl.full[it % kStages], (it / kStages) & 1, P.wait_limit_ns, &ctl.abort)) return false;
        tc_fence_after();
        const uint64_t a = sw128_desc(kaddr + (it % kStages) * 2 * kTileBytes), b = sw128_desc(qaddr);
#pragma unroll
        for (int j = 0; j < kHeadDim / 32; ++j)   // 32 elements of d a step: 32 bytes of a row
          tc_mma_e4m3(tmem, a + 2 * j, b + 2 * j, C::kIdescS, j > 0);
        tc_commit(&ctl.s_full);
        return true;
      };
      bool ok = scores(0, true);
      for (int it = 0; ok && it < n; ++it) {
        if (!mbar_wait(&ctl.p_full, it & 1, P.wait_limit_ns, &ctl.abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t vaddr = kaddr + (it % kStages) * 2 * kTileBytes + kTileBytes;
#pragma unroll
        for (int j = 0; j < kTileKeys / 32; ++j)   // 32 tokens a step: four 8-row groups of V, of P
          tc_mma_e4m3(tmem + C::kOCol, sw128_mn_desc(vaddr + 4096u * j, kTileBytes, 1024),
                      plain_mn_desc(paddr + 512u * j, 128, 16 * kTileKeys), C::kIdescO, j > 0);
        tc_commit(&ctl.empty[it % kStages]);
        tc_commit(&ctl.o_full);
        if (it + 1 < n) {
          ++x;
          const bool fresh = x == at.first + at.tiles;
          if (fresh) at.next(P, blocks);
          ok = scores(it + 1, fresh);
        }
      }
      if (!ok) {
        fail();
        tc_commit(&ctl.drain);   // what was issued ends before TMEM is given back
        mbar_wait(&ctl.drain, 0, P.wait_limit_ns, &ctl.never);
      }
    }
  } else {
    // ------------------------------------------------------------ softmax: a token, then a column, a thread
    // sequences without a token: their rows are zeros
    for (int r = blockIdx.x; r < P.n_seq; r += gridDim.x)
      if (Walk::length(P, r) == 0)
        for (int i = 0; i < P.q_tokens * P.c.hq; ++i) {
          const int64_t tok = static_cast<int64_t>(r) * P.q_tokens + i / P.c.hq;
          P.out[tok * P.o_st + (i % P.c.hq) * P.o_sh + tid] = 0;
          if (P.lse && tid == 0) P.lse[tok * P.c.hq + i % P.c.hq] = -INFINITY;
        }
    if (works) {
      const uint32_t quad = static_cast<uint32_t>(warp) << 21;   // this warp's TMEM lanes
      uint8_t* qbuf = smem + C::kQ;
      uint8_t* pbuf = smem + C::kP;
      uint32_t met = 0;
      // all 128 threads; what each wrote to shared memory before is seen behind it
      const auto meet = [&]() -> bool {
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.meet);
        return warp_wait(&ctl.meet, met++ & 1u, P.wait_limit_ns, &ctl.abort);
      };
      // Query rows of a block as two e4m3 pieces, K-major with the 128-byte swizzle. 128 / R threads a
      // row, R elements each.
      const auto load_q = [&](const Walk& w, int parity) {
        constexpr int kPer = R, kLanes = 128 / R;
        const int i = tid / kLanes, c = tid % kLanes * kPer, row = w.rb * R + i;
        uint32_t x[kPer / 2];
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) x[j] = 0;
        if (row < rows) {
          const int64_t tok = static_cast<int64_t>(w.r) * P.q_tokens + row / P.c.group;
          const uint16_t* src = P.q + tok * P.q_st + (w.h * P.c.group + row % P.c.group) * P.q_sh + c;
          if constexpr (kPer == 4) {
            const uint2 y = __ldg(reinterpret_cast<const uint2*>(src));
            x[0] = y.x, x[1] = y.y;
          } else {
#pragma unroll
            for (int j = 0; j < kPer / 8; ++j) {
              const uint4 y = __ldg(reinterpret_cast<const uint4*>(src) + j);
              x[4 * j] = y.x, x[4 * j + 1] = y.y, x[4 * j + 2] = y.z, x[4 * j + 3] = y.w;
            }
          }
        }
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) m = max(m, max(x[j] & 0x7fffu, (x[j] >> 16) & 0x7fffu));
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const bool finite = m < 0x7f80u;
        const float scale = __uint_as_float(finite ? piece_scale(m) : 0u);
        uint32_t hi[kPer / 4], lo[kPer / 4];
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
          const float a = finite ? __uint_as_float(x[j] << 16) * scale : 0.f;
          const float b = finite ? __uint_as_float(x[j] & 0xffff0000u) * scale : 0.f;
          const uint32_t two = e4m3x2(a, b);
          const float2 f = e4m3x2_values(two);
          const uint32_t rest = e4m3x2((a - f.x) * 16.f, (b - f.y) * 16.f);
          hi[j / 2] = j % 2 ? hi[j / 2] | two << 16 : two;
          lo[j / 2] = j % 2 ? lo[j / 2] | rest << 16 : rest;
        }
        const auto put = [&](int n, const uint32_t* v) {
          uint8_t* dst = qbuf + n * kHeadDim + (((c >> 4) ^ (n & 7)) << 4) + (c & 15);
          if constexpr (kPer == 4) {
            *reinterpret_cast<uint32_t*>(dst) = v[0];
          } else if constexpr (kPer == 8) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(v[0], v[1]);
          } else {
            *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
          }
        };
        put(i, hi);
        put(R + i, lo);
        // a row with an infinity or a NaN: every logit NaN
        if (tid % kLanes == 0) ctl.qs[parity][i] = finite ? P.alpha * __frcp_rn(scale) : __uint_as_float(0x7fc00000u);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.q_full);
      };

      Walk at;
      at.seek(P, blocks, ctl.first_r, ctl.base, x0);
      if constexpr (2 * R < C::kNs)   // columns behind the pieces: zeros, once
        for (int i = tid; i < (C::kNs - 2 * R) * kHeadDim / 4; i += 128)
          reinterpret_cast<uint32_t*>(qbuf + 2 * R * kHeadDim)[i] = 0;
      int part = 0;
      load_q(at, 0);
      bool ok = meet();
      float m[R], l[R], acc[R];
      int seen[R];   // tokens that the row sees
      int nan_from = INT32_MAX;   // the first position with a NaN in this column, among those not all rows see
      const auto begin = [&]() {
#pragma unroll
        for (int i = 0; i < R; ++i) {
          m[i] = -INFINITY;
          l[i] = acc[i] = 0.f;
          const int row = at.rb * R + i;
          seen[i] = row < rows ? at.len - P.q_tokens + row / P.c.group + 1 : 0;
        }
        nan_from = INT32_MAX;
      };
      if (ok) begin();
      long long x = x0, part0 = x0;
      const int n = static_cast<int>(x1 - x0);
      for (int it = 0; ok && it < n; ++it, ++x) {
        const int st = it % kStages;
        const int pos = static_cast<int>(x - at.first) * kTileKeys + tid;
        if (!warp_wait(&ctl.full[st], (it / kStages) & 1, P.wait_limit_ns, &ctl.abort)) {
          ok = false;
          break;
        }
        const int pg = tid >> P.c.page_shift;
        const uint32_t have = ctl.pages[st];
        const bool held = (have >> pg & 1u) && pos < at.len;
        const float ks = ctl.ks[st][pg];
        float vtop = 0.f;
#pragma unroll
        for (int j = 0; j < kMostTilePages; ++j) vtop = fmaxf(vtop, ctl.vs[st][j]);
        // the largest scale of the tile's values comes out of the sums; a token keeps the rest (at most 1)
        const float vrest = held && vtop > 0.f ? ctl.vs[st][pg] * __frcp_rn(vtop) * 256.f : 0.f;
        if (!warp_wait(&ctl.s_full, it & 1, P.wait_limit_ns, &ctl.abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        float s[C::kNs];
        if constexpr (C::kNs == 16) tmem_ld16(tmem + quad, s);
        else tmem_ld32(tmem + quad, s);
        tmem_wait_ld(s);
        float w[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float y = fmaf(s[R + i], 0.0625f, s[i]) * ctl.qs[part & 1][i] * ks;
          w[i] = held && pos < seen[i] ? y : -INFINITY;
        }
        float* red = &ctl.red[it & 1][warp][0];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float top = warp_max(w[i]);
          if (lane == i) red[i] = top;
        }
        if (!meet()) {
          ok = false;
          break;
        }
        float keep[R];   // exp(old maximum - new)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float top = fmaxf(fmaxf(ctl.red[it & 1][0][i], ctl.red[it & 1][1][i]),
                                  fmaxf(ctl.red[it & 1][2][i], ctl.red[it & 1][3][i]));
          const float mn = fmaxf(m[i], top), ref = mn == -INFINITY ? 0.f : mn;
          keep[i] = ex2(m[i] - ref);
          m[i] = mn;
          const float p = ex2(w[i] - ref);
          l[i] = fmaf(l[i], keep[i], p);
          w[i] = w[i] == -INFINITY ? 0.f : p * vrest;
        }
        // three e4m3 pieces of each probability: column k R + i of the token's row
        uint32_t out[C::kNp / 4];
#pragma unroll
        for (int i = 0; i < C::kNp / 4; ++i) out[i] = 0;
#pragma unroll
        for (int i = 0; i < R; i += 2) {
          float a = w[i], b = w[i + 1];
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const uint32_t two = e4m3x2(a, b);
            out[(k * R + i) / 4] |= two << (8 * ((k * R + i) % 4));
            if (k < 2) {
              const float2 f = e4m3x2_values(two);
              a = (a - f.x) * 16.f;
              b = (b - f.y) * 16.f;
            }
          }
        }
#pragma unroll
        for (int c = 0; c < C::kNp / 16; ++c)
          *reinterpret_cast<uint4*>(pbuf + c * (16 * kTileKeys) + tid * 16) =
              make_uint4(out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]);
        const int tile_end = pos - tid + kTileKeys;
        const bool all = have == (0xffu >> (kMostTilePages - (kTileKeys >> P.c.page_shift))) && tile_end <= at.len;
        const bool some = P.q_tokens > 1 && tile_end > at.len - P.q_tokens + 1;
        if (!all || some) {
          uint8_t* v = smem + static_cast<size_t>(st) * 2 * kTileBytes + kTileBytes;
          if (!held) {
            // a probability of 0 does not undo a NaN: rows without a token are zeros
#pragma unroll
            for (int j = 0; j < kHeadDim / 16; ++j) reinterpret_cast<uint4*>(v + tid * kHeadDim)[j] = make_uint4(0, 0, 0, 0);
          }
          if (some) {
            // nor may a NaN value that later rows see reach the earlier ones: it is taken out here, and
            // given to the rows that see it when the part ends
            const int t0 = max(at.len - P.q_tokens + 1 - (pos - tid), 0), t1 = min(at.len - (pos - tid), kTileKeys);
            for (int t = t0; t < t1; ++t) {
              uint8_t* at8 = v + t * kHeadDim + (((tid >> 4) ^ (t & 7)) << 4) + (tid & 15);
              if ((have >> (t >> P.c.page_shift) & 1u) && (*at8 & 0x7f) == 0x7f) {
                nan_from = min(nan_from, pos - tid + t);
                *at8 = 0;
              }
            }
          }
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.p_full);
        const bool part_ends = x + 1 == x1 || x + 1 == at.first + at.tiles;
        Walk then = at;
        if (part_ends && x + 1 < x1) {
          // the next block's rows while the tensor cores work (the scores of this one are done)
          then.next(P, blocks);
          load_q(then, (part + 1) & 1);
        }
        if (!warp_wait(&ctl.o_full, it & 1, P.wait_limit_ns, &ctl.abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        float o[C::kNp];
        if constexpr (C::kNp == 16) {
          tmem_ld16(tmem + C::kOCol + quad, o);
        } else {
          tmem_ld32(tmem + C::kOCol + quad, o);
          if constexpr (C::kNp == 48) tmem_ld16(tmem + C::kOCol + 32 + quad, o + 32);
        }
        tmem_wait_ld(o);
        tc_fence_before();
        const float back = vtop * (1.f / 256.f);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float y = fmaf(fmaf(o[2 * R + i], 0.0625f, o[R + i]), 0.0625f, o[i]);
          acc[i] = fmaf(y, back, acc[i] * keep[i]);
        }
        if (!part_ends) continue;

        // ---------------------------------------------------------- the end of a part
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (seen[i] > nan_from) acc[i] = __uint_as_float(0x7fc00000u);
        // row sums over the tokens' threads
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
          for (int o2 = 16; o2 > 0; o2 >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o2);
          if (lane == i) ctl.red[(it + 1) & 1][warp][i] = l[i];   // (the next tile writes there behind a meet)
        }
        if (!meet()) {
          ok = false;
          break;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float(*red4)[R] = ctl.red[(it + 1) & 1];
          l[i] = (red4[0][i] + red4[1][i]) + (red4[2][i] + red4[3][i]);
        }
        bool write = true;
        const long long end = at.first + at.tiles;
        if (part0 != at.first || x + 1 != end) {
          // one of several parts: leave it for the CTA that finishes last
          const int w0 = static_cast<int>(((at.first + 1) * ctas + total - 1) / total) - 1;
          const int w1 = static_cast<int>((end * ctas + total - 1) / total) - 1;
          const auto slot = [&](int w) {   // a part that starts where the CTA does, or a later one
            return P.partial + (static_cast<int64_t>(w) * 2 + (w == w0 && share(w) != at.first ? 1 : 0)) * kAttendPartWords;
          };
          float* dst = slot(blockIdx.x);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            __stcg(dst + i * kHeadDim + tid, acc[i]);
            if (tid == i) {
              __stcg(dst + R * kHeadDim + i, m[i]);
              __stcg(dst + R * kHeadDim + R + i, l[i]);
            }
          }
          __threadfence();
          if (!meet()) {
            ok = false;
            break;
          }
          if (tid == 0) ctl.last = atomicInc(P.arrive + w0, static_cast<unsigned>(w1 - w0)) == static_cast<unsigned>(w1 - w0);
          if (!meet()) {
            ok = false;
            break;
          }
          write = ctl.last != 0;
          if (write) {
            __threadfence();
#pragma unroll
            for (int i = 0; i < R; ++i) {
              m[i] = -INFINITY;
              l[i] = acc[i] = 0.f;
            }
            for (int wk = w0; wk <= w1; ++wk) {
              const float* src = slot(wk);
#pragma unroll
              for (int i = 0; i < R; ++i) {
                const float pm = __ldcg(src + R * kHeadDim + i), pl = __ldcg(src + R * kHeadDim + R + i);
                const float po = __ldcg(src + i * kHeadDim + tid);
                const float mn = fmaxf(m[i], pm), ref = mn == -INFINITY ? 0.f : mn;
                const float f = ex2(m[i] - ref), g = ex2(pm - ref);
                l[i] = l[i] * f + pl * g;
                acc[i] = acc[i] * f + po * g;
                m[i] = mn;
              }
            }
          }
        }
        if (write) {
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const int row = at.rb * R + i;
            if (row < rows) {
              const int64_t tok = static_cast<int64_t>(at.r) * P.q_tokens + row / P.c.group;
              const int hq = at.h * P.c.group + row % P.c.group;
              const bool none = l[i] == 0.f;   // (a NaN sum is not: its row is NaN)
              P.out[tok * P.o_st + hq * P.o_sh + tid] = none ? 0 : to_bf16(acc[i] / l[i]);
              if (P.lse && tid == 0)
                P.lse[tok * P.c.hq + hq] = none ? -INFINITY : (m[i] == -INFINITY ? 0.f : m[i]) * 0.69314718056f +
                                                                   lg2(l[i]) * 0.69314718056f;
            }
          }
        }
        if (x + 1 < x1) {
          at = then;
          ++part;
          part0 = x + 1;
          begin();
          ok = meet();   // the next block's scales are there, and this one's sums have been read
        }
      }
      if (!ok && lane == 0) fail();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    tmem_dealloc(tmem, C::kTmemCols);
  }
}

template <int R>
cudaError_t attend_rows(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  constexpr size_t smem = attend_smem<R>();
  static_assert(smem <= 113 * 1024, "two CTAs an SM");
  cudaError_t e = cudaFuncSetAttribute(cache_attend_kernel<R>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  // no more CTAs than there can be tiles
  const int64_t blocks = (p.q_tokens * p.c.group + R - 1) / R;
  const int64_t tiles = ((static_cast<int64_t>(p.c.max_pages) << p.c.page_shift) + kTileKeys - 1) / kTileKeys;
  const int64_t most = static_cast<int64_t>(kAttendCtas) * c.sms;
  const int64_t want = tiles >= most ? most : tiles * p.n_seq * p.c.heads * blocks;
  return launch_after_previous(cache_attend_kernel<R>, dim3(static_cast<unsigned>(want < most ? want : most)),
                               dim3(kAttendThreads), smem, stream, c.tm_k, c.tm_v, p);
}

}  // namespace

cudaError_t launch_cache_attend(const kve_cache& c, const AttendParams& p, cudaStream_t stream) {
  const int rows = p.q_tokens * p.c.group;
  if (rows <= 4) return attend_rows<4>(c, p, stream);
  if (rows <= 8) return attend_rows<8>(c, p, stream);
  return attend_rows<16>(c, p, stream);
}

}  // namespace kve
