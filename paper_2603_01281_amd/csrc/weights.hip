// seka_attention_weights: how much attention every cached token gets from new tokens.
//
//   W_out[b, h, j] = decay W_in[b, h, j] + sum over heads g of the group and the last `window` new tokens i that see j
//                    of exp(scale q_{i,g} . k_j - lse_{i,g})
//
// A wave holds 16 KT keys in registers and passes the rows by (new token i and head g are row i G + g), 16 at a time:
// S (rows x keys) = Q K^T, so that a lane has one key and four rows of every product, adds up its exponentials in place, and the
// sums cross lanes once, behind the last row.  No scores, no atomics: the result does not depend on scheduling.
// SHARE: the waves of a workgroup take the same keys and every fourth tile of rows, and join their sums in LDS; otherwise each
// wave has keys of its own.
#include <algorithm>

#include "paged.h"

namespace seka {
namespace {

constexpr int kWtWaves = 4, kWtTiles = 4;       // waves, tiles of 16 keys per wave

template <typename T> struct WtMath;
template <> struct WtMath<uint16_t> {
  typedef bf16x8 frag;
  static constexpr int CH = 1;
  __device__ static __forceinline__ void mma(f32x4 (&acc)[1], const frag& a, const frag& b) {
    acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc[0], 0, 0, 0);
  }
};
template <> struct WtMath<float> {
  typedef f32x4 frag;
  static constexpr int CH = 4;            // four short chains of sums
  __device__ static __forceinline__ void mma(f32x4 (&acc)[4], const frag& a, const frag& b) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc[e], 0, 0, 0);
  }
};

template <typename T, int D, bool SHARE>
__global__ __launch_bounds__(64 * kWtWaves, 2) void weights_kernel(WeightsArgs a) {
  using M = WtMath<T>;
  typedef typename M::frag frag;
  constexpr int NF = D * sizeof(T) / 64, KT = kWtTiles, KEYS = 16 * KT;      // fragments of a row: 64 bytes over four lanes each
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  __shared__ float sm[SHARE ? kWtWaves : 1][SHARE ? KEYS : 1];

  const int b = blockIdx.z, h = blockIdx.y, G = a.Hq / a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const ChunkExtent e = chunk_extent(a.r, a.c, b);
  const int kbase = SHARE ? blockIdx.x * KEYS : (blockIdx.x * kWtWaves + wave) * KEYS;
  if (kbase >= e.len) return;              // SHARE: the whole workgroup; otherwise no barrier follows

  // ---- keys: lane (key 16 kt + l16, bytes 64 f + 16 grp); behind the last one it is repeated ----
  frag kf[KT][NF];
  size_t home[KT];                         // of this lane's keys in the weights
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int j = min(kbase + 16 * kt + l16, e.len - 1);
    const int page = page_of(a.c, b, j), slot = j & ((1 << a.c.shift) - 1);
    home[kt] = (((size_t)page * a.Hkv + h) << a.c.shift) + slot;
    const char* kp = static_cast<const char*>(a.c.K) + (((((size_t)page << a.c.shift) + slot) * a.Hkv + h) * D) * sizeof(T) + 16 * grp;
#pragma unroll
    for (int f = 0; f < NF; ++f) kf[kt][f] = __builtin_bit_cast(frag, *reinterpret_cast<const u32x4*>(kp + 64 * f));
  }

  // ---- rows that count and see the first of these keys ----
  const int ctx = e.len - e.n;
  const int i_lo = max(max(e.n - a.window, kbase - ctx), 0);
  const int rows = e.n * G, r_lo = min(i_lo, e.n) * G;
  const float c2 = a.scale * 1.4426950408889634f;
  float sum[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) sum[kt] = 0.f;

  frag qn[NF];
  float lse_n = INFINITY;
  int i_n = 0;
  auto fetch = [&](int r0) __attribute__((always_inline)) {
    const int row = r0 + l16;
    const bool ok = row < rows;
    const int i = ok ? row / G : 0, hq = h * G + (ok ? row - i * G : 0);
    i_n = i;
    lse_n = INFINITY;                      // rows that do not exist or see nothing: exp(. - inf) = 0
    const char* qp = static_cast<const char*>(a.Q) + ((size_t)(e.row0 + i) * a.Hq + hq) * D * sizeof(T) + 16 * grp;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      u32x4 v = {0, 0, 0, 0};
      if (ok) v = *reinterpret_cast<const u32x4*>(qp + 64 * f);
      qn[f] = __builtin_bit_cast(frag, v);
    }
    if (ok) {
      const float x = a.lse[(size_t)hq * a.r.total + e.row0 + i];
      lse_n = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
    }
  };
  const int step = SHARE ? 16 * kWtWaves : 16;
  int r0 = r_lo + (SHARE ? 16 * wave : 0);
  if (r0 < rows) fetch(r0);
  for (; r0 < rows; r0 += step) {
    frag q[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) q[f] = qn[f];
    float lse2[4];
    int last[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) lse2[x] = __shfl(lse_n, 4 * grp + x);
    const bool masked = ctx + r0 / G < kbase + KEYS - 1;
    if (masked) {
#pragma unroll
      for (int x = 0; x < 4; ++x) last[x] = ctx + __shfl(i_n, 4 * grp + x);
    }
    if (r0 + step < rows) fetch(r0 + step);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f32x4 acc[M::CH];
#pragma unroll
      for (int c = 0; c < M::CH; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < NF; ++f) M::mma(acc, q[f], kf[kt][f]);
#pragma unroll
      for (int half = M::CH / 2; half; half /= 2)
#pragma unroll
        for (int c = 0; c < half; ++c) acc[c] += acc[c + half];
      float p[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) p[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[0][x], c2, -lse2[x]));
      if (masked) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (kbase + 16 * kt + l16 > last[x]) p[x] = 0.f;
      }
      sum[kt] += (p[0] + p[1]) + (p[2] + p[3]);
    }
  }

#pragma unroll
  for (int kt = 0; kt < KT; ++kt) sum[kt] = groups_sum(sum[kt]);
  if (SHARE) {
    if (grp == 0) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) sm[wave][16 * kt + l16] = sum[kt];
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sum[kt] = 0.f;
#pragma unroll
      for (int w = 0; w < kWtWaves; ++w) sum[kt] += sm[SHARE ? w : 0][SHARE ? 16 * kt + l16 : 0];
    }
  }
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
    if (grp == 0 && kbase + 16 * kt + l16 < e.len)
      a.c.W[home[kt]] = sum[kt] + (a.W_in ? a.decay * a.W_in[home[kt]] : 0.f);
}

template <typename T, int D>
hipError_t launch(const WeightsArgs& a, hipStream_t s) {
  // few rows: the keys are the work, every wave has its own
  const bool share = (long long)std::min(std::min(a.r.max_q, a.window), a.r.total) * (a.Hq / a.Hkv) > 64;
  const int keys = 16 * kWtTiles * (share ? 1 : kWtWaves);
  const dim3 grid((a.c.cap + keys - 1) / keys, a.Hkv, a.r.B), block(64 * kWtWaves);
  if (share) hipLaunchKernelGGL((weights_kernel<T, D, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((weights_kernel<T, D, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_weights(const WeightsArgs& a, int D, int dtype, hipStream_t s) {
  if (dtype == SEKA_BF16) return D == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return D == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace seka
