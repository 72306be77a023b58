// Attention over the paged 8-bit cache: rows (t, g) of a sequence and cache head h, the query heads
// h*G + g at positions len - T + t, over the visible tokens i < len - T + t + 1 of its pages:
//   l_i = (q . c_i) s_page / sqrt(d),   out = sum_i softmax(l)_i v_i,   lse = ln sum_i exp(l_i).
#include "kve_internal.h"
#include "kve_ptx.cuh"

namespace kve {
namespace {

constexpr int kAttendThreads = 128;

__device__ __forceinline__ float e4m3_value(uint8_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(c)));
  float f;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.f32.f16 %0, a;\n}" : "=f"(f) : "r"(h));
  return f;
}

// One CTA a query row, 128 tokens at a time: thread i the logit of token i, then thread d column d of
// the value product, with the running maximum and sum of the softmax.
__global__ void __launch_bounds__(kAttendThreads) cache_attend_kernel(const __grid_constant__ AttendParams P) {
  wait_previous_kernel();
  __shared__ float q[kHeadDim], w[kAttendThreads];
  __shared__ float red[2][4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hq = blockIdx.x % P.c.hq, h = hq / P.c.group;
  const int tok = blockIdx.x / P.c.hq, r = tok / P.q_tokens, t = tok % P.q_tokens;
  const int cap = P.c.max_pages << P.c.page_shift;
  int len = __ldg(P.lens + r);
  if ((len < 0 || len > cap) && tid == 0) atomicOr(P.err, kErrCheck);
  len = min(max(len, 0), cap);
  const int seen = len - P.q_tokens + t + 1;
  const uint16_t x = P.q[static_cast<int64_t>(tok) * P.q_st + hq * P.q_sh + tid];
  q[tid] = __uint_as_float(static_cast<uint32_t>(x) << 16);
  const bool finite = __syncthreads_and((x & 0x7f80u) != 0x7f80u);
  const int32_t* row = P.table + static_cast<int64_t>(r) * P.c.max_pages;
  float m = -INFINITY, sum = 0.f, acc = 0.f;
  for (int i0 = 0; i0 < seen; i0 += kAttendThreads) {
    const int i = i0 + tid;
    float l = -INFINITY;
    if (i < seen) {
      const int page = __ldg(row + (i >> P.c.page_shift));
      if (page < 0 || page >= P.c.num_pages) {
        atomicOr(P.err, kErrCheck);
      } else {
        const int64_t b = static_cast<int64_t>(page) * P.c.heads + h;
        const uint8_t* k = P.c.k + (b * P.c.page + (i & (P.c.page - 1))) * kHeadDim;
        float a = 0.f;
        for (int d = 0; d < kHeadDim; ++d) a = fmaf(q[d], e4m3_value(k[d]), a);
        l = a * P.alpha * P.c.k_scale[b];
      }
    }
    float top = l;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) red[0][warp] = top;
    __syncthreads();
    const float mn = fmaxf(fmaxf(fmaxf(m, red[0][0]), fmaxf(red[0][1], red[0][2])), red[0][3]);
    const float ref = mn == -INFINITY ? 0.f : mn;
    float p = l == -INFINITY ? 0.f : exp2f(l - ref);
    w[tid] = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) p += __shfl_xor_sync(0xffffffffu, p, o);
    if (lane == 0) red[1][warp] = p;
    __syncthreads();
    const float f = m == -INFINITY ? 0.f : exp2f(m - ref);
    sum = sum * f + ((red[1][0] + red[1][1]) + (red[1][2] + red[1][3]));
    acc *= f;
    const int n = min(seen - i0, kAttendThreads);
    for (int j = 0; j < n; ++j) {
      const int page = __ldg(row + ((i0 + j) >> P.c.page_shift));
      if (page < 0 || page >= P.c.num_pages) continue;
      const int64_t b = static_cast<int64_t>(page) * P.c.heads + h;
      acc = fmaf(w[j] * P.c.v_scale[b],
                 e4m3_value(P.c.v[(b * P.c.page + ((i0 + j) & (P.c.page - 1))) * kHeadDim + tid]), acc);
    }
    m = mn;
    __syncthreads();
  }
  float o = sum > 0.f || sum != sum ? acc / sum : 0.f;
  float lse = sum > 0.f || sum != sum ? (m + log2f(sum)) * 0.69314718056f : -INFINITY;
  if (!finite && seen > 0) o = lse = __uint_as_float(0x7fc00000u);
  uint32_t bits = __float_as_uint(o);
  bits = o != o ? 0x7fc0u : (bits + 0x7fffu + (bits >> 16 & 1u)) >> 16;
  P.out[static_cast<int64_t>(tok) * P.o_st + hq * P.o_sh + tid] = static_cast<uint16_t>(bits);
  if (P.lse && tid == 0) P.lse[static_cast<int64_t>(tok) * P.c.hq + hq] = lse;
}

}  // namespace

cudaError_t launch_cache_attend(const kve_cache&, const AttendParams& p, cudaStream_t stream) {
  return launch_after_previous(cache_attend_kernel, dim3(static_cast<unsigned>(p.n_seq * p.q_tokens * p.c.hq)),
                               dim3(kAttendThreads), 0, stream, p);
}

}  // namespace kve
