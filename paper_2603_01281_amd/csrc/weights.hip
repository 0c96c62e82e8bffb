// seka_attention_weights: how much attention every cached token gets from new tokens.
//
//   W_out[b, h, j] = decay W_in[b, h, j] + sum over heads g of the group and the last `window` new tokens i that see j
//                    of exp(scale q_{i,g} . k_j - lse_{i,g})
//
// Rows: new token i and head g are row i G + g.  S (rows x keys) = Q K^T in tiles of 16 x 16: a lane has one key and four rows of
// every product, adds up its exponentials in place, and the sums cross lanes once, behind the last row.  No scores in
// memory, no atomics: the result does not depend on scheduling.
//
// Few rows (generation): HBM-bound, every key is read once.  weights_stream_kernel holds the rows and streams the keys as whole rows
// through a wave-private LDS tile, a block ahead, over ranges that are cut as for the attention itself (paged.h, plan_item).
// Many rows: bound by the vector unit (an exponential takes it four times as long as a multiplication; 96 cycles per tile of 16 x 16
// against 64 of the matrix pipe at D = 128).  weights_block_kernel holds 32 keys per wave (fp32, D = 128: 16) in registers and passes the rows by, 64 or 128 at a
// time through LDS for all its waves; two groups of waves have the same keys and take half of the rows each (one wave per SIMD had
// nothing to hide its latencies behind: a chunk of 1000 over 8192, 32 / 8 heads, 142 us).  weights_share_kernel, where those would leave compute units idle: 64 keys per workgroup,
// every wave its share of the rows, straight from the caches; the waves' sums are joined in LDS.
// One token of 24 requests of up to 8192, 32 / 8 heads, D = 128: 35 us, 4.1 TB/s; 1000 over 8192 beside one: 82 us, 0.77 PFLOP/s.
#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace seka {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
constexpr int kWtWaves = 4, kWtThreads = 64 * kWtWaves;
// tiles of 16 keys that a wave holds (four of fp32 rows of 512 bytes did not fit its registers)
template <typename T, int D> constexpr int wt_tiles() { return D * sizeof(T) > 256 ? 2 : 4; }
// rows that pass through LDS at a time (no more than two 16-byte pieces to a thread, where there are 128 registers)
template <typename T, int D, int NW> constexpr int wt_block_rows() { return D * sizeof(T) > 256 || (NW == 4 && D * sizeof(T) == 256) ? 64 : 128; }
constexpr int kWtGroups = 2;                // groups of waves with the same keys, each with its share of those rows
template <typename T, int D> constexpr int wt_block_tiles() { return wt_tiles<T, D>() / 2; }      // 128 registers: four waves to a SIMD

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

// Scores of a tile: rows 4 grp + x of the lane's key.
template <typename T, int NF>
__device__ __forceinline__ f32x4 wt_tile(const typename WtMath<T>::frag (&q)[NF], const typename WtMath<T>::frag (&k)[NF]) {
  using M = WtMath<T>;
  f32x4 acc[M::CH];
#pragma unroll
  for (int c = 0; c < M::CH; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int f = 0; f < NF; ++f) M::mma(acc, q[f], k[f]);
#pragma unroll
  for (int half = M::CH / 2; half; half /= 2)
#pragma unroll
    for (int c = 0; c < half; ++c) acc[c] += acc[c + half];
  return acc[0];
}

// A row's log-sum-exp in units of the exponent; rows that saw nothing count nothing: exp(. - inf) = 0.
__device__ __forceinline__ float wt_reference(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

// One tile of rows against the wave's keys: all products, then all exponentials, so that one key tile's hide behind another's.
template <bool MASKED, typename T, int NF, int KT>
__device__ __forceinline__ void wt_rows(const typename WtMath<T>::frag (&q)[NF], const typename WtMath<T>::frag (&kf)[KT][NF], const float (&ref)[4],
                                        const int (&last)[4], int kbase, float c2, float (&sum)[KT]) {
  const int l16 = threadIdx.x & 15;
  f32x4 s[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) s[kt] = wt_tile<T, NF>(q, kf[kt]);
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    float p[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) p[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][x], c2, -ref[x]));
    if (MASKED) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (kbase + 16 * kt + l16 > last[x]) p[x] = 0.f;
    }
    sum[kt] += (p[0] + p[1]) + (p[2] + p[3]);
  }
}

// The keys have arrived: a wait for them inside the loop over the rows would wait for the next rows too.
template <int KT, int NF, typename F>
__device__ __forceinline__ void wt_arrived(F (&kf)[KT][NF]) {
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int f = 0; f < NF; ++f) asm volatile("" : "+v"(kf[kt][f]));
}

// ---- few rows ------------------------------------------------------------------------------------------------------------

template <typename T, int D, int RT>
__global__ __launch_bounds__(kWtThreads, 2) void weights_stream_kernel(WeightsArgs a) {
  typedef typename WtMath<T>::frag frag;
  constexpr int RB = D * sizeof(T), NF = RB / 64;                       // bytes of a row, fragments of it: 64 bytes over four lanes each
  constexpr int BK = sizeof(T) == 2 ? 32 : 16, KT = BK / 16;
  constexpr int CPR = RB / 16, RPI = 64 / CPR, NV = BK / RPI;           // 16-byte pieces per row, rows per load, loads per block
  constexpr int LD = RB + 16;                                           // LDS row stride (bytes): 16 rows at one piece, spread over all banks
  __shared__ __attribute__((aligned(16))) unsigned char smem[kWtWaves * BK * LD];

  ChunkItem it;
  if (!plan_item(a.r, a.c, a.p, blockIdx.x, it)) return;
  int k0, k1;
  plan_range(a.p, it, k0, k1);
  const int h = blockIdx.y, G = a.Hq / a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const int ctx = it.e.len - it.e.n;
  const int row_lo = max(it.e.n - a.window, 0) * G, rows = it.e.n * G;
  unsigned char* tile = smem + wave * BK * LD;

  frag q[RT][NF];
  float ref[RT][4];
  int last[RT][4];                         // last key that the row sees
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = row_lo + 16 * rt + l16;
    const bool ok = row < rows;
    const int i = ok ? row / G : 0, hq = h * G + (ok ? row % G : 0);
    const char* qp = static_cast<const char*>(a.Q) + ((size_t)(it.e.row0 + i) * a.Hq + hq) * RB + 16 * grp;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      u32x4 v = {0, 0, 0, 0};
      if (ok) v = *reinterpret_cast<const u32x4*>(qp + 64 * f);
      q[rt][f] = __builtin_bit_cast(frag, v);
    }
    float r = INFINITY;
    if (ok) r = wt_reference(a.lse[(size_t)hq * a.r.total + it.e.row0 + i]);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      ref[rt][x] = __shfl(r, 4 * grp + x);
      last[rt][x] = ctx + __shfl(i, 4 * grp + x);
    }
  }
  const int all_see = ctx + row_lo / G;    // keys up to here are seen by every row
  const float c2 = a.scale * 1.4426950408889634f;

  const uint32_t row_bytes = (uint32_t)a.Hkv * RB;
  const uint32_t lane_off = (uint32_t)(lane / CPR) * row_bytes + 16u * (lane % CPR);
  const char* Kh = static_cast<const char*>(a.c.K) + (size_t)h * RB;
  const int slots = (1 << a.c.shift) - 1;
  u32x4 kr[NV];
  float w_in = 0.f;
  size_t home = 0, home_next = 0;          // of key kb + lane, lane < BK
  PageWindow<BK, kWtWaves> win;
  int block = 0;
  auto fetch = [&](int kb) __attribute__((always_inline)) {
    if (block == win.left) {
      win.load(a.c, it.b, kb, k1);
      block = 0;
    }
    const int at = block * win.per_block;
    ++block;
    if (kb + BK <= k1) {
#pragma unroll
      for (int x = 0; x < NV; ++x) {       // the RPI <= 8 rows of a load lie in one page
        const int page = __builtin_amdgcn_readlane(win.entry, at + (win.per_block > 1 ? (RPI * x) >> a.c.shift : 0));
        const size_t off = (((size_t)page << a.c.shift) + ((kb + RPI * x) & slots)) * row_bytes;
        kr[x] = *reinterpret_cast<const u32x4*>(Kh + off + lane_off);
      }
    } else {                               // rows behind the last key repeat it
#pragma unroll
      for (int x = 0; x < NV; ++x) {
        const int key = min(kb + RPI * x + lane / CPR, k1 - 1);
        const int page = __shfl(win.entry, at + (win.per_block > 1 ? (key - kb) >> a.c.shift : 0));
        kr[x] = *reinterpret_cast<const u32x4*>(Kh + (((size_t)page << a.c.shift) + (key & slots)) * row_bytes + 16u * (lane % CPR));
      }
    }
    const int key = min(kb + (lane & (BK - 1)), k1 - 1);
    const int page = __shfl(win.entry, at + (win.per_block > 1 ? (key - kb) >> a.c.shift : 0));
    home_next = (((size_t)page * a.Hkv + h) << a.c.shift) + (key & slots);
    if (a.W_in) w_in = a.W_in[home_next];
  };

  int kb = k0 + wave * BK;
  if (kb < k1) {
    win.load(a.c, it.b, kb, k1);
    fetch(kb);
  }
  for (; kb < k1; kb += kWtWaves * BK) {
#pragma unroll
    for (int x = 0; x < NV; ++x) *reinterpret_cast<u32x4*>(tile + (RPI * x + lane / CPR) * LD + 16 * (lane % CPR)) = kr[x];
    asm volatile("" ::: "memory");         // (a wave's LDS operations execute in program order)
    const float w = w_in;
    home = home_next;
    if (kb + kWtWaves * BK < k1) fetch(kb + kWtWaves * BK);
    float sum[KT];
    frag k[KT][NF];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sum[kt] = 0.f;
#pragma unroll
      for (int f = 0; f < NF; ++f) k[kt][f] = *reinterpret_cast<const frag*>(tile + (16 * kt + l16) * LD + 64 * f + 16 * grp);
    }
    const bool masked = kb + BK - 1 > all_see;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (masked) wt_rows<true, T, NF, KT>(q[rt], k, ref[rt], last[rt], kb, c2, sum);
      else wt_rows<false, T, NF, KT>(q[rt], k, ref[rt], last[rt], kb, c2, sum);
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) sum[kt] = groups_sum(sum[kt]);
    asm volatile("" ::: "memory");         // the tile is rewritten behind these reads
    if (lane < BK && kb + lane < k1) a.c.W[home] = (KT == 2 && grp == 1 ? sum[KT - 1] : sum[0]) + (a.W_in ? a.decay * w : 0.f);
  }
}

// ---- many rows -----------------------------------------------------------------------------------------------------------

// A wave's keys: lane (key 16 kt + l16, bytes 64 f + 16 grp); behind the last one it is repeated.  home: this lane's keys in the weights.
template <typename T, int D, int NF, int KT>
__device__ __forceinline__ void wt_keys(const WeightsArgs& a, const ChunkExtent& e, int b, int h, int kbase, typename WtMath<T>::frag (&kf)[KT][NF],
                                        size_t (&home)[KT]) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int j = min(kbase + 16 * kt + l16, e.len - 1);
    const int page = page_of(a.c, b, j), slot = j & ((1 << a.c.shift) - 1);
    home[kt] = (((size_t)page * a.Hkv + h) << a.c.shift) + slot;
    const char* kp = static_cast<const char*>(a.c.K) + (((((size_t)page << a.c.shift) + slot) * a.Hkv + h) * D) * sizeof(T) + 16 * grp;
#pragma unroll
    for (int f = 0; f < NF; ++f) kf[kt][f] = __builtin_bit_cast(typename WtMath<T>::frag, *reinterpret_cast<const u32x4*>(kp + 64 * f));
  }
}

// NW: waves of a group.
template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * kWtGroups * NW, 4) void weights_block_kernel(WeightsArgs a) {
  typedef typename WtMath<T>::frag frag;
  constexpr int kWtBlockWaves = NW, kWtBlockThreads = 64 * kWtGroups * NW;
  constexpr int RB = D * sizeof(T), NF = RB / 64, KT = wt_block_tiles<T, D>(), KEYS = 16 * KT, kWtRows = wt_block_rows<T, D, NW>();
  constexpr int CPR = RB / 16, NL = (kWtRows * CPR + kWtBlockThreads - 1) / kWtBlockThreads;    // pieces of a row, loads per thread and turn
  constexpr int LD = RB + 16;
  __shared__ __attribute__((aligned(16))) unsigned char rows_lds[2][kWtRows * LD];
  __shared__ __attribute__((aligned(16))) float ref_lds[2][kWtRows];
  __shared__ __attribute__((aligned(16))) int last_lds[2][kWtRows];

  const int b = blockIdx.z, h = blockIdx.y, G = a.Hq / a.Hkv, tid = threadIdx.x;
  const int lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) % kWtBlockWaves, group = __builtin_amdgcn_readfirstlane(tid >> 6) / kWtBlockWaves;
  const ChunkExtent e = chunk_extent(a.r, a.c, b);
  const int kfirst = blockIdx.x * kWtBlockWaves * KEYS;       // of the workgroup
  if (kfirst >= e.len) return;                           // workgroup-uniform
  const int kbase = kfirst + wave * KEYS;
  frag kf[KT][NF];
  size_t home[KT];
  wt_keys<T, D, NF, KT>(a, e, b, h, min(kbase, e.len - 1), kf, home);

  // rows that count and see the workgroup's first key
  const int ctx = e.len - e.n;
  const int i_lo = max(max(e.n - a.window, kfirst - ctx), 0);
  const int rows = e.n * G, r_lo = min(i_lo, e.n) * G;
  const float c2 = a.scale * 1.4426950408889634f;
  float sum[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) sum[kt] = 0.f;

  u32x4 next[NL];
  float ref_next = INFINITY;
  int last_next = 0;
  auto fetch = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      const int c = tid + kWtBlockThreads * x, row = min(r0 + min(c / CPR, kWtRows - 1), rows - 1);
      const int i = row / G, hq = h * G + row - i * G;
      next[x] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.Q) + ((size_t)(e.row0 + i) * a.Hq + hq) * RB + 16 * (c % CPR));
    }
    if (tid < kWtRows) {
      const int row = r0 + tid, i = min(row, rows - 1) / G, hq = h * G + min(row, rows - 1) - i * G;
      const float x = a.lse[(size_t)hq * a.r.total + e.row0 + i];
      ref_next = row < rows ? wt_reference(x) : INFINITY;
      last_next = ctx + i;
    }
  };
  auto place = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      const int c = tid + kWtBlockThreads * x;
      if (kWtRows * CPR % kWtBlockThreads == 0 || c < kWtRows * CPR) *reinterpret_cast<u32x4*>(rows_lds[buf] + (c / CPR) * LD + 16 * (c % CPR)) = next[x];
    }
    if (tid < kWtRows) {
      ref_lds[buf][tid] = ref_next;
      last_lds[buf][tid] = last_next;
    }
  };
  if (r_lo < rows) {
    fetch(r_lo);
    place(0);
  }
  wt_arrived(kf);
  __syncthreads();
  int buf = 0;
  for (int r0 = r_lo; r0 < rows; r0 += kWtRows, buf ^= 1) {
    if (r0 + kWtRows < rows) fetch(r0 + kWtRows);
    // this group's tiles of the rows: every second one, of those that hold any (all 64 or 128 for a request with one token: fp32, 14 requests of up to
    // 18 new tokens over 13524, 8 / 2 heads, 45 us, without 35)
    auto turn = [&](auto masked, auto whole) __attribute__((always_inline)) {
      constexpr int NT = kWtRows / 16 / kWtGroups;
      constexpr int AHEAD = sizeof(T) == 2 && decltype(whole)::value;      // a tile's rows are read while the one before is worked on (fp32: no registers left)
      frag q[1 + AHEAD][NF];
      auto read = [&](int r16) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < NF; ++f) q[r16 & AHEAD][f] = *reinterpret_cast<const frag*>(rows_lds[buf] + (16 * (kWtGroups * r16 + group) + l16) * LD + 64 * f + 16 * grp);
      };
      auto work = [&](int r16) __attribute__((always_inline)) {
        const int first = 16 * (kWtGroups * r16 + group) + 4 * grp;
        const f32x4 ref4 = *reinterpret_cast<const f32x4*>(&ref_lds[buf][first]);
        float ref[4];
        int last[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          ref[x] = ref4[x];
          last[x] = decltype(masked)::value ? last_lds[buf][first + x] : 0;
        }
        wt_rows<decltype(masked)::value, T, NF, KT>(q[r16 & AHEAD], kf, ref, last, kbase, c2, sum);
      };
      if constexpr (decltype(whole)::value) {
        if (AHEAD) read(0);
#pragma unroll
        for (int r16 = 0; r16 < NT; ++r16) {
          if (r16 + AHEAD < NT) read(r16 + AHEAD);
          work(r16);
        }
      } else {
        const int n = ((rows - r0 + 15) / 16 - group + kWtGroups - 1) / kWtGroups;
#pragma nounroll
        for (int r16 = 0; r16 < n; ++r16) {
          read(r16);
          work(r16);
        }
      }
    };
    const bool masks = ctx + r0 / G < kbase + KEYS - 1;  // (all wave-uniform)
    if (kbase >= e.len) {}                               // no keys of its own
    else if (r0 + kWtRows > rows) turn(std::true_type{}, std::false_type{});
    else masks ? turn(std::true_type{}, std::true_type{}) : turn(std::false_type{}, std::true_type{});
    if (r0 + kWtRows < rows) place(buf ^ 1);             // read by nobody since the barrier before
    __syncthreads();
  }
  // the second group's sums to the first (the rows' area is free behind the last barrier)
  float* sm = reinterpret_cast<float*>(rows_lds) + wave * KEYS;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    sum[kt] = groups_sum(sum[kt]);
    if (group == 1 && grp == 0) sm[16 * kt + l16] = sum[kt];
  }
  __syncthreads();
  if (group == 1 || grp != 0) return;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
    if (kbase + 16 * kt + l16 < e.len) a.c.W[home[kt]] = sum[kt] + sm[16 * kt + l16] + (a.W_in ? a.decay * a.W_in[home[kt]] : 0.f);
}

template <typename T, int D>
__global__ __launch_bounds__(kWtThreads, 2) void weights_share_kernel(WeightsArgs a) {
  typedef typename WtMath<T>::frag frag;
  constexpr int RB = D * sizeof(T), NF = RB / 64, KT = wt_tiles<T, D>(), KEYS = 16 * KT;
  __shared__ float sm[kWtWaves][KEYS];
  const int b = blockIdx.z, h = blockIdx.y, G = a.Hq / a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const ChunkExtent e = chunk_extent(a.r, a.c, b);
  const int kbase = blockIdx.x * KEYS;
  if (kbase >= e.len) return;              // workgroup-uniform
  frag kf[KT][NF];
  size_t home[KT];
  wt_keys<T, D, NF, KT>(a, e, b, h, kbase, kf, home);

  const int ctx = e.len - e.n;
  const int i_lo = max(max(e.n - a.window, kbase - ctx), 0);
  const int rows = e.n * G, r_lo = min(i_lo, e.n) * G;
  const float c2 = a.scale * 1.4426950408889634f;
  float sum[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) sum[kt] = 0.f;
  frag qn[NF];
  float ref_n = INFINITY;
  int i_n = 0;
  auto fetch = [&](int r0) __attribute__((always_inline)) {
    const int row = r0 + l16, at = min(row, rows - 1), i = at / G, hq = h * G + at - i * G;
    const char* qp = static_cast<const char*>(a.Q) + ((size_t)(e.row0 + i) * a.Hq + hq) * RB + 16 * grp;
#pragma unroll
    for (int f = 0; f < NF; ++f) qn[f] = __builtin_bit_cast(frag, *reinterpret_cast<const u32x4*>(qp + 64 * f));
    const float x = a.lse[(size_t)hq * a.r.total + e.row0 + i];
    ref_n = row < rows ? wt_reference(x) : INFINITY;
    i_n = i;
  };
  int r0 = r_lo + 16 * wave;
  wt_arrived(kf);
  if (r0 < rows) fetch(r0);
  for (; r0 < rows; r0 += 16 * kWtWaves) {
    frag q[NF];
    float ref[4];
    int last[4];
#pragma unroll
    for (int f = 0; f < NF; ++f) q[f] = qn[f];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      ref[x] = __shfl(ref_n, 4 * grp + x);
      last[x] = ctx + __shfl(i_n, 4 * grp + x);
    }
    if (r0 + 16 * kWtWaves < rows) fetch(r0 + 16 * kWtWaves);
    if (ctx + r0 / G < kbase + KEYS - 1) wt_rows<true, T, NF, KT>(q, kf, ref, last, kbase, c2, sum);
    else wt_rows<false, T, NF, KT>(q, kf, ref, last, kbase, c2, sum);
  }
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    sum[kt] = groups_sum(sum[kt]);
    if (grp == 0) sm[wave][16 * kt + l16] = sum[kt];
  }
  __syncthreads();
  if (wave != 0 || grp != 0) return;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWtWaves; ++w) s += sm[w][16 * kt + l16];
    if (kbase + 16 * kt + l16 < e.len) a.c.W[home[kt]] = s + (a.W_in ? a.decay * a.W_in[home[kt]] : 0.f);
  }
}

template <typename T, int D>
hipError_t launch(WeightsArgs a, hipStream_t s) {
  const long long rows = (long long)std::min(std::min(a.r.max_q, a.window), a.r.total) * (a.Hq / a.Hkv);
  const dim3 threads(kWtThreads);
  constexpr int kFew = D * sizeof(T) > 256 ? 32 : 64;      // rows that the streaming kernel's registers hold
  if (rows <= kFew) {
    a.p.R = 0;
    a.p.G = a.Hq / a.Hkv;
    a.p.slots_log2 = 0;
    while ((1 << a.p.slots_log2) * a.Hkv < 2048) ++a.p.slots_log2;
    a.p.least = 8;
    a.p.max_splits = std::max(1, (a.c.cap + 255) / 256);
    const int items = (int)std::min((long long)a.r.B + (1 << a.p.slots_log2), (long long)a.r.B * a.p.max_splits);
    const dim3 grid(items, a.Hkv);
    if (rows <= 16) hipLaunchKernelGGL((weights_stream_kernel<T, D, 1>), grid, threads, 0, s, a);
    else if (rows <= 32) hipLaunchKernelGGL((weights_stream_kernel<T, D, 2>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((weights_stream_kernel<T, D, kFew / 16>), grid, threads, 0, s, a);
    return hipGetLastError();
  }
  constexpr int KEYS = 16 * wt_tiles<T, D>();
  // Groups of eight waves where the rows are many, and their passage through LDS serves more keys; else of four, two workgroups to a compute unit.  us, eight /
  // four: 4000 rows, 8192 keys, 32 / 8 heads 82 / 91; 1248 rows of ten requests of up to 1919 48.9 / 36.4; 289 rows, ten of up to 10141, 32 / 32 218 / 175.
  constexpr int kWave = 16 * wt_block_tiles<T, D>();
  const int waves = rows > 2048 ? 8 : 4, blocks = (a.c.cap + kWave * waves - 1) / (kWave * waves);
  const dim3 grid(blocks, a.Hkv, a.r.B), block(64 * kWtGroups * waves);
  const bool many = (long long)blocks * a.Hkv * a.r.B >= 256;
  if (many && waves == 8) hipLaunchKernelGGL((weights_block_kernel<T, D, 8>), grid, block, 0, s, a);
  else if (many) hipLaunchKernelGGL((weights_block_kernel<T, D, 4>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((weights_share_kernel<T, D>), dim3((a.c.cap + KEYS - 1) / KEYS, a.Hkv, a.r.B), threads, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_weights(const WeightsArgs& a, int D, int dtype, hipStream_t s) {
  if (dtype == SEKA_BF16) return D == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return D == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace seka
