// Rotary positions: the frequencies and handles of the C interface, and the kernel that turns rows by them.
//
// Pair j of a row at position n turns by the angle n f_j: (a, b) -> A (a cos - b sin, b cos + a sin). The gradient of that
// is the same turn backwards (the transpose), and so is the inverse where A = 1.
//
// Bound by HBM: 256 bytes read and 256 written a row; the turns of a token are computed once for all of its heads that a CTA
// has, in shared memory, and nothing is read for them but the position.
#include <cmath>
#include <cstring>
#include <new>

#include "kve_rotary.cuh"

namespace kve {
namespace {

constexpr int kRotateThreads = 256;

// 16,411 tokens of 40 heads (336 MB, half of each head turns) take 51.4 us of 50.3 at a copy's rate, the window rows of 32 layers
// (17 MB) 5.1 of 2.5, which is the launch, positions, rows. Two rows a lane in flight and 32 warps an SM; four rows and 24 warps took
// 52.1 and 5.8, two and 40 52.1 and 5.3, two and 48 (spills) 58.3 and 6.6.
__global__ void __launch_bounds__(kRotateThreads, 4) rotate_kernel(const __grid_constant__ RotateParams P) {
  wait_previous_kernel();
  __shared__ __align__(16) float2 turns[kTurnTokens * kMaxPairs];
  rotate_tile<kRotateThreads, 2>(P, blockIdx.x, turns);
  allow_next_kernel();
}

// f / (2 pi) without its whole turns, in units of 2^-64 to the nearest (|f| < 2^62: within an eighth of a unit more). f = m 2^e with
// an integer m of 53 bits, times 1 / (2 pi) in 128 bits; a division in 64-bit floating point would be off by 2^-56 of a turn, which a
// position of 2^31 makes 2^-25.
uint64_t units_of_turn(double f) {
  constexpr uint64_t kHigh = 0x28be60db9391054aull, kLow = 0x7f09d5f47d4d3770ull;   // 2^128 / (2 pi)
  int e = 0;
  const uint64_t m = static_cast<uint64_t>(std::ldexp(std::frexp(std::fabs(f), &e), 53));
  using Wide = unsigned __int128;
  const Wide low = static_cast<Wide>(m) * kLow, high = static_cast<Wide>(m) * kHigh + (low >> 64);
  const uint64_t w[4] = {static_cast<uint64_t>(low), static_cast<uint64_t>(high), static_cast<uint64_t>(high >> 64), 0};
  // the product's bits from 2^shift on
  const int shift = 117 - e;
  uint64_t units = 0;
  if (shift <= 0) {
    units = shift > -64 ? w[0] << -shift : 0;
  } else if (shift < 192) {
    const int i = shift / 64, by = shift % 64;
    units = by == 0 ? w[i] : w[i] >> by | w[i + 1] << (64 - by);
    const int half = shift - 1;
    units += w[half / 64] >> half % 64 & 1u;
  }
  return f < 0.0 ? 0 - units : units;
}

}  // namespace

cudaError_t launch_rotate(const RotateParams& params, cudaStream_t stream) {
  RotateParams p = params;
  const int64_t tiles = cut_rotate<kRotateThreads>(p);
  return launch_after_previous(rotate_kernel, dim3(static_cast<unsigned>(tiles)), dim3(kRotateThreads), 0, stream, p);
}

}  // namespace kve

extern "C" {

kve_status kv_evict_rotary_frequencies(int32_t kind, int32_t rotary_dim, double base, double factor, double original_length,
                                       double low_turns, double high_turns, double* frequencies, double* amplitude) {
  const double two_pi = 6.283185307179586476925;
  if (!frequencies || !amplitude || kind < KVE_ROTARY_NONE || kind > KVE_ROTARY_YARN) return KVE_EINVAL;
  if (rotary_dim < 16 || rotary_dim > kve::kHeadDim || rotary_dim % 16) return KVE_EINVAL;
  if (!std::isfinite(base) || base <= 1.0) return KVE_EINVAL;
  if (kind != KVE_ROTARY_NONE && (!std::isfinite(factor) || factor < 1.0)) return KVE_EINVAL;
  const bool by_turns = kind == KVE_ROTARY_PARTS || kind == KVE_ROTARY_YARN;
  if (by_turns && !(std::isfinite(original_length) && original_length >= 1.0 && std::isfinite(high_turns) && low_turns > 0.0 &&
                    high_turns > low_turns))
    return KVE_EINVAL;
  const double n = rotary_dim;
  if (kind == KVE_ROTARY_NTK) base *= std::pow(factor, n / (n - 2.0));
  if (!std::isfinite(base)) return KVE_EINVAL;
  *amplitude = kind == KVE_ROTARY_YARN ? 1.0 + 0.1 * std::log(factor) : 1.0;
  double first = 0.0, last = 0.0;
  if (kind == KVE_ROTARY_YARN) {   // the pairs that make high_turns and low_turns within the original length
    const double per = n / (2.0 * std::log(base));
    first = std::fmax(std::floor(per * std::log(original_length / (two_pi * high_turns))), 0.0);
    last = std::fmin(std::ceil(per * std::log(original_length / (two_pi * low_turns))), n - 1.0);
  }
  for (int j = 0; j < rotary_dim / 2; ++j) {
    const double f = std::pow(base, -2.0 * j / n);
    double keep = 1.0;
    if (kind == KVE_ROTARY_LINEAR) keep = 0.0;
    if (kind == KVE_ROTARY_PARTS) keep = (original_length * f / two_pi - low_turns) / (high_turns - low_turns);
    if (kind == KVE_ROTARY_YARN) keep = 1.0 - (j - first) / std::fmax(last - first, 0.001);
    keep = std::fmin(std::fmax(keep, 0.0), 1.0);
    frequencies[j] = kind == KVE_ROTARY_NONE || kind == KVE_ROTARY_NTK ? f : keep * f + (1.0 - keep) * (f / factor);
  }
  return KVE_OK;
}

kve_status kv_evict_rotary_create(int32_t head_dim, int32_t rotary_dim, int32_t interleaved, const double* frequencies,
                                  double amplitude, kve_rotary** out) {
  if (!out) return KVE_EINVAL;
  *out = nullptr;
  if (!frequencies || head_dim != kve::kHeadDim || rotary_dim < 16 || rotary_dim > head_dim || rotary_dim % 16 ||
      (interleaved != 0 && interleaved != 1) || !std::isfinite(amplitude) || std::fabs(amplitude) > 1e30)
    return KVE_EINVAL;
  for (int j = 0; j < rotary_dim / 2; ++j)
    if (!std::isfinite(frequencies[j])) return KVE_EINVAL;
  kve_rotary* h = new (std::nothrow) kve_rotary;
  if (!h) return KVE_ENOMEM;
  std::memset(h, 0, sizeof(*h));
  for (int j = 0; j < rotary_dim / 2; ++j) {
    // high 2^32 + low, with low signed
    const uint64_t units = kve::units_of_turn(frequencies[j]);
    h->table.turns[j].x = static_cast<uint32_t>(units);
    h->table.turns[j].y = static_cast<uint32_t>((units >> 32) + (units >> 31 & 1u));
  }
  h->table.amplitude = static_cast<float>(amplitude);
  h->table.pairs = rotary_dim / 2;
  h->table.interleaved = interleaved;
  *out = h;
  return KVE_OK;
}

void kv_evict_rotary_destroy(kve_rotary* rotary) { delete rotary; }

kve_status kv_evict_rotary_apply(const kve_rotary* rotary, const uint16_t* x, const int64_t* x_strides, uint16_t* out,
                                 const int64_t* out_strides, int32_t heads, const int32_t* positions, int64_t n_tokens,
                                 int32_t transpose, void* stream) {
  if (!rotary || heads < 1 || n_tokens < 0 || n_tokens >= (int64_t(1) << 31) / heads || (transpose != 0 && transpose != 1))
    return KVE_EINVAL;
  if (n_tokens > 0 && (!x || !out || !positions)) return KVE_EINVAL;
  const auto aligned = [](const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; };
  if (!aligned(x, 16) || !aligned(out, 16) || !aligned(positions, 4)) return KVE_EINVAL;
  kve::RotateParams p;
  std::memset(&p, 0, sizeof(p));
  if (!kve::row_strides(x_strides, heads, &p.x_st, &p.x_sh) || !kve::row_strides(out_strides, heads, &p.o_st, &p.o_sh))
    return KVE_EINVAL;
  if (!kve::rows_apart(n_tokens, p.o_st, heads, p.o_sh)) return KVE_EINVAL;
  if (x == out && (p.x_st != p.o_st || p.x_sh != p.o_sh)) return KVE_EINVAL;
  if (n_tokens == 0) return KVE_OK;
  const int device = kve::place_of(out);
  int current = -1;
  if (device == kve::kHostMemory || (device >= 0 && (cudaGetDevice(&current) != cudaSuccess || current != device)))
    return KVE_EINVAL;
  p.r = rotary->table;
  p.x = x;
  p.out = out;
  p.positions = positions;
  p.n_tokens = n_tokens;
  p.heads = heads;
  p.transpose = transpose;
  return kve::launch_rotate(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KVE_OK : KVE_ECUDA;
}

}  // extern "C"
