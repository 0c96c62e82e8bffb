// seka_attention_chunk: new tokens of a batch of requests attend to their caches of pages, bf16.
//
//   s_ij = scale q_i . k_j for j <= len - n + i;   O_i = sum_j softmax(s_i)_j v_j;   lse_i = log sum_j exp(s_ij)
//
// Rows: new token i and head g of a KV head's group are row i G + g, so that all of a group's queries share every key read.
// A workgroup takes R = 16 RT rows of one request and KV head and a range of its keys (paged.h, plan_item); its four waves take
// 32-key blocks in turn and never synchronise before they merge.
//   S^T (keys x rows)  = K q^T       A = K rows from LDS, B = queries in registers
//   O^T (D x rows)    += V^T P^T     A = V^T by transposing LDS reads, B = P^T straight from the S^T accumulators
// Keys and values are fetched as whole rows into registers, a block ahead, and pass through a wave-private LDS tile.
// HBM-bound at generation: one token of 24 requests of up to 8192, 32 / 8 heads, D = 128, 277 MB in 64 us, 4.4 TB/s (a large copy 5.2); ranges end
// up to a block apart and a second kernel of 4 us joins them.  Small calls are two launches' latency: 7 us in one range, 10 in several.
// Many rows take the kernels whose waves have rows of their own (pipe_plan below).
#include <algorithm>

#include "chunk_pipe.h"
#include "chunk_rows.h"
#include "compute_units.h"

namespace seka {
namespace {

typedef __attribute__((address_space(3))) s16x4* row_lds_s16x4_ptr;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

template <int D, int RT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void chunk_rows_bf16_kernel(ChunkArgs a) {
  constexpr int BK = 32, R = 16 * RT;
  // LDS row strides (elements): 16 rows of K at one 16-byte column, and 16 rows x 32 bytes of V, spread over all banks
  constexpr int LDK = D + 8, LDV = D + 16, OLD = D + 4;
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int CPR = D / 8, RPI = 64 / CPR, NV = BK / RPI;     // 16-byte pieces per row, rows per load, loads per block
  constexpr int kTileBytes = BK * LDV * 2, kMergeBytes = 16 * OLD * 4;
  constexpr int kAreaBytes = kTileBytes > kMergeBytes ? kTileBytes : kMergeBytes;
  __shared__ __attribute__((aligned(16))) unsigned char smem[NW * kAreaBytes];
  __shared__ float sm_ml[NW][16][2];

  ChunkItem it;
  const bool exists = plan_item(a.r, a.c, a.p, blockIdx.x, it);
  row_describe(a, exists, it);
  if (!exists) return;                     // workgroup-uniform
  int k0, k1;
  plan_range(a.p, it, k0, k1);
  const int h = blockIdx.y, G = a.p.G;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const int nrows = it.e.n * G, ctx = it.e.len - it.e.n;
  uint16_t* tile = reinterpret_cast<uint16_t*>(smem + wave * kAreaBytes);

  // ---- queries: lane (row 16 rt + l16, d = 32 ks + 8 grp ..) ----
  bf16x8 qf[RT][KS];
  int last[RT];                            // last key that this lane's row sees
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = it.rc * R + 16 * rt + l16;
    const bool ok = row < nrows;
    const int i = ok ? row / G : 0, g = ok ? row % G : 0;
    last[rt] = ok ? ctx + i : -1;
    const uint16_t* qp = static_cast<const uint16_t*>(a.Q) + ((size_t)(it.e.row0 + i) * a.Hq + h * G + g) * D + 8 * grp;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 v = {0, 0, 0, 0};
      if (ok) v = *reinterpret_cast<const u32x4*>(qp + 32 * ks);
      qf[rt][ks] = __builtin_bit_cast(bf16x8, v);
    }
  }
  const int all_see = ctx + it.rc * R / G; // keys up to here are seen by every row

  float m[RT], l[RT];
  f32x4 o[DT][RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kRowLow;
    l[rt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = a.scale * 1.4426950408889634f;

  const uint32_t row_bytes = (uint32_t)a.Hkv * D * 2;
  const uint32_t lane_off = (uint32_t)(lane / CPR) * row_bytes + 16u * (lane % CPR);
  const char* Kh = static_cast<const char*>(a.c.K) + (size_t)h * D * 2;
  const char* Vh = static_cast<const char*>(a.c.V) + (size_t)h * D * 2;
  const int slots = (1 << a.c.shift) - 1;
  u32x4 kr[NV], vr[NV];
  PageWindow<BK, NW> win;
  int block = 0;                           // of the window
  auto fetch = [&](auto nt, int kb) __attribute__((always_inline)) {
    constexpr bool NT = decltype(nt)::value;
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
        kr[x] = paged_load<NT>(reinterpret_cast<const u32x4*>(Kh + off + lane_off));
        vr[x] = paged_load<NT>(reinterpret_cast<const u32x4*>(Vh + off + lane_off));
      }
    } else {                               // rows behind the last key repeat it
#pragma unroll
      for (int x = 0; x < NV; ++x) {
        const int key = min(kb + RPI * x + lane / CPR, k1 - 1);
        const int page = __shfl(win.entry, at + (win.per_block > 1 ? (key - kb) >> a.c.shift : 0));
        const size_t off = (((size_t)page << a.c.shift) + (key & slots)) * row_bytes + 16u * (lane % CPR);
        kr[x] = paged_load<NT>(reinterpret_cast<const u32x4*>(Kh + off));
        vr[x] = paged_load<NT>(reinterpret_cast<const u32x4*>(Vh + off));
      }
    }
  };

  // NT where all caches of the call outgrow the last-level cache: keys then leave room for what is read again
  auto run = [&](auto nt) __attribute__((always_inline)) {
    int kb = k0 + wave * BK;
    if (kb < k1) {
      win.load(a.c, it.b, kb, k1);
      fetch(nt, kb);
    }
    row_arrived(qf);
    for (; kb < k1; kb += NW * BK) {
      // (a wave's LDS operations execute in program order; the fences are for the compiler)
#pragma unroll
      for (int x = 0; x < NV; ++x) *reinterpret_cast<u32x4*>(tile + (RPI * x + lane / CPR) * LDK + 8 * (lane % CPR)) = kr[x];
      asm volatile("" ::: "memory");
      f32x4 sc[2][RT];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) sc[kt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const bf16x8 kf = *reinterpret_cast<const bf16x8*>(tile + (16 * kt + l16) * LDK + 32 * ks + 8 * grp);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) sc[kt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rt][ks], sc[kt][rt], 0, 0, 0);
        }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int x = 0; x < NV; ++x) *reinterpret_cast<u32x4*>(tile + (RPI * x + lane / CPR) * LDV + 8 * (lane % CPR)) = vr[x];
      asm volatile("" ::: "memory");
      const int kb_next = kb + NW * BK;
      if (kb_next < k1) fetch(nt, kb_next);      // on their way during the softmax

      bf16x8 pb[RT];
      const bool masked = kb + BK - 1 > all_see || kb + BK > k1;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = sc[e >> 2][rt][e & 3] * c2;
        if (masked) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (kb + 16 * (e >> 2) + 4 * grp + (e & 3) > last[rt]) t[e] = -INFINITY;
        }
        float top = t[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, t[e]);
        top = groups_max(top);
        const bool raise = top > m[rt] + kRowSlack;
        if (__any(raise)) {                  // rare behind the first blocks
          const float f = raise ? __builtin_amdgcn_exp2f(m[rt] - top) : 1.f;
          if (raise) m[rt] = top;
          l[rt] *= f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[dt][rt] *= f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(t[e] - m[rt]);
          l[rt] += p;                        // of the probabilities before their rounding
          pb[rt][e] = (__bf16)p;
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        // lane: d = 16 dt + l16, slot e <-> key 16 (e / 4) + 4 grp + e % 4, as in the score accumulators
        const uint16_t* p = tile + (4 * grp + (l16 >> 2)) * LDV + 16 * dt + 4 * (l16 & 3);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((row_lds_s16x4_ptr)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((row_lds_s16x4_ptr)(p + 16 * LDV));
        const bf16x8 vf = __builtin_shufflevector(__builtin_bit_cast(bf16x4, lo), __builtin_bit_cast(bf16x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[dt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[rt], o[dt][rt], 0, 0, 0);
      }
      asm volatile("" ::: "memory");         // the tile is rewritten behind these reads
    }
  };
  if (it.streams) run(std::true_type{});
  else run(std::false_type{});

  // ---- merge the waves, 16 rows at a time; lane (row l16, grp) holds O[row][16 dt + 4 grp + i] ----
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float lt = groups_sum(l[rt]);
    __syncthreads();                       // the tiles, or the merge area of the rows before, are free
    float* mo = reinterpret_cast<float*>(smem) + wave * 16 * OLD;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(mo + l16 * OLD + 16 * dt + 4 * grp) = o[dt][rt];
    if (grp == 0) {
      sm_ml[wave][l16][0] = m[rt];
      sm_ml[wave][l16][1] = lt;
    }
    __syncthreads();
    merge_waves<uint16_t, D, NW>(a, it, h, it.rc * R + 16 * rt, reinterpret_cast<const float*>(smem), sm_ml);
  }
}

template <int D, int NW>
void launch_rows(const ChunkArgs& a, const RowPlan& r, hipStream_t s) {
  const dim3 grid(r.items, a.Hkv), block(64 * NW);
  if (r.rows16 == 1) hipLaunchKernelGGL((chunk_rows_bf16_kernel<D, 1, NW>), grid, block, 0, s, a);
  else if (r.rows16 == 2) hipLaunchKernelGGL((chunk_rows_bf16_kernel<D, 2, NW>), grid, block, 0, s, a);
  else if constexpr (D == 64) hipLaunchKernelGGL((chunk_rows_bf16_kernel<D, 4, 4>), grid, dim3(256), 0, s, a);
}

template <int D>
hipError_t launch_rows(const ChunkArgs& a, const RowPlan& r, hipStream_t s) {
  if (r.waves == 8) launch_rows<D, 8>(a, r, s);
  else launch_rows<D, 4>(a, r, s);
  launch_chunk_merge<uint16_t, D>(a, r.items, r.rows, s);
  return hipGetLastError();
}

constexpr int kOneRange = 1024;          // cached tokens, bf16: no more than these are one range

// Rows per workgroup, ranges and the bounds of both, from what the host knows: B requests, `total` new tokens of which no request
// has more than max_q, caches of up to S tokens.
RowPlan row_plan(int B, int S, int Hq, int Hkv, int D, int dtype, int total, int max_q) {
  RowPlan r;
  const int G = Hq / Hkv, blocks = (S + 31) / 32;
  const bool bf16 = dtype == SEKA_BF16;
  const long long rows = (long long)std::min(max_q, total) * G;
  r.p.G = G;
  r.p.least = bf16 ? 8 : 4;                // 256 tokens, 128: a block of every wave of eight
  const long long ranges = std::max(1, std::min(kMaxRanges, (blocks + r.p.least - 1) / r.p.least));
  auto chunks_of = [&](int R) { return std::min(((long long)total * G) / R + B, 0x3fffffffll); };
  // as many tiles of 16 rows as there are, up to two (D = 64: four), but no more than leave two workgroups for every compute unit.  Four at
  // D = 128 need the registers of two waves: 10 new tokens over 24967, 32 / 8 heads, 60.1 us, in two chunks of two tiles 32.5.
  r.rows16 = rows <= 16 ? 1 : rows <= 32 || D == 128 ? 2 : 4;
  while (r.rows16 > 1 && chunks_of(16 * r.rows16) * ranges * Hkv < 512) r.rows16 /= 2;
  r.p.R = 16 * r.rows16;
  r.rows = (int)std::min(rows, (long long)r.p.R);
  const long long chunks = chunks_of(r.p.R);
  // eight waves to a workgroup where the keys are few: a range is then half as long a chain
  const bool few = r.rows16 <= 2 && chunks * blocks * Hkv <= 256 * 8 * 2 && chunks * Hkv <= 256;
  r.waves = few ? 8 : 4;
  // two workgroups of four waves to a compute unit, about, or one of eight
  r.p.slots_log2 = 0;
  while ((1 << r.p.slots_log2) * Hkv < (few ? 256 : 512)) ++r.p.slots_log2;
  r.p.max_splits = (int)ranges;
  // and no second kernel where a wave has no more than four blocks, eight of four waves (bf16, 37 requests of up to 24 over 526, 32 / 4 heads, D = 64:
  // 27.4 us in ranges, 12.8 in one each; fp32, 777 tokens in one range: 14.5 us, in ranges 9.9)
  if (bf16 ? S <= kOneRange : few && S <= 512) r.p.max_splits = 1;
  r.p.streams = (long long)(300e6 / (2.0 * 32 * Hkv * D * (bf16 ? 2 : 4)));
  // sum over chunks of ceil(blocks / L) <= T / L + chunks with T / L <= slots, and no more than every chunk in all its ranges
  r.items = (int)std::min(chunks + (1 << r.p.slots_log2), chunks * r.p.max_splits);
  return r;
}

int compute_units() {
  static PerDeviceCount cus;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  return cus.of(dev, [](int d) {
    int n = 0;
    return hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, d) == hipSuccess && n > 0 ? n : 256;
  });
}

// Products of a call's rows with S keys each, in flops, from which on long chunks go to the kernel whose waves have rows of their own; bf16, and its caches
// that the kernel of few rows takes in one range.  us, few rows / pipelined: 2.2e9 three of up to 153 over 7358, 5 / 5 heads, D = 64, 28.3 / 27.5; 3.2e9 three of up
// to 11 over 27872, 32 / 4, D = 64, 29.6 / 32.5; 4.9e9 four of up to 194 over 1515, 32 / 8, 37.3 / 32.4; 1.5e10 four of up to 491 over 1354, 24 / 8, 56.3 / 39.3;
// in one range: 4.9e9 three of up to 942 over 996, 8 / 2, 19.4 / 29.7; 6.8e9 63 of up to 73 over 376, 32 / 8, 32.7 / 37.4; 8.1e9 24 of up to 379 over 379, 30.3 / 26.9.
constexpr double kPipeLeastFlops = 3.5e9, kPipeLeastFlopsShort = 7.5e9;
// And fp32, at D = 64 and 128.  us, few rows / blocks: D = 64, 7.7e8 n=75 S=5039 8 / 2 heads 24.9 / 47.4, 1.2e9 ten of up to 26 over 1465 43.0 / 35.8, 3e9
// n=388 S=934 73.6 / 53.4; D = 128, 5.7e9 four of up to 85 over 14804 5 / 5 heads 91.1 / 107, 1.2e10 ten of up to 58 over 9466 147 / 149, 1.6e10 n=422
// S=2284 196 / 159, 2.3e10 six of up to 65 over 6984 196 / 162.
constexpr double kBlockLeastFlops64 = 1e9, kBlockLeastFlops128 = 1.2e10;

// Whether a call's chunks go to a kernel whose waves have rows of their own, and how: more rows per KV head than four tiles of 16, and, bf16, a
// cache whose page numbers fit beside the tiles in LDS (4 bytes for every page of S tokens).
bool pipe_plan(int S, int Hq, int Hkv, int D, int dtype, int shift, int total, int max_q, PipeChunkPlan* out) {
  const int G = Hq / Hkv;
  const bool bf16 = dtype == SEKA_BF16;
  if ((long long)std::min(max_q, total) * G <= 64) return false;
  if (4.0 * D * total * Hq * S <= (bf16 ? (S <= kOneRange ? kPipeLeastFlopsShort : kPipeLeastFlops) : D == 64 ? kBlockLeastFlops64 : kBlockLeastFlops128)) return false;
  out->width = std::max(1, (bf16 ? 1 : 2) * compute_units() / Hkv);      // workgroups to a compute unit
  out->smem = !bf16 ? 0 : attention_bf16_pipe_smem_bytes(D, 0, false, 1, PipeBf16::WAVES) + (((size_t)S >> shift) + 2) * sizeof(int);
  out->cuts = (size_t)2 * out->width * Hkv * (bf16 ? PipeBf16::ROWS : PipeF32::ROWS) * (D + 4) * sizeof(float);      // behind the states, two per workgroup
  out->workspace = out->cuts + (size_t)out->width * sizeof(int4);
  return out->smem <= 160 * 1024;
}

}  // namespace

hipError_t launch_chunk_bf16(const ChunkArgs& a, int D, const RowPlan& r, hipStream_t s) {
  return D == 128 ? launch_rows<128>(a, r, s) : launch_rows<64>(a, r, s);
}

size_t row_states(const RowPlan& r, int Hkv, int D) { return r.p.max_splits > 1 ? (size_t)r.items * Hkv * r.p.R * (D + 4) * sizeof(float) : 0; }

// (the larger need: which kernel runs depends on the page size too)
size_t chunk_workspace_bytes(int B, int S, int Hq, int Hkv, int D, int dtype, int total, int max_q) {
  const RowPlan r = row_plan(B, S, Hq, Hkv, D, dtype, total, max_q);
  const size_t rows = row_states(r, Hkv, D) + (size_t)r.items * sizeof(int4);
  PipeChunkPlan p;
  return pipe_plan(S, Hq, Hkv, D, dtype, 16, total, max_q, &p) ? std::max(rows, p.workspace) : rows;
}

hipError_t launch_chunk(ChunkArgs a, int D, int dtype, int S, hipStream_t s) {
  PipeChunkPlan p;
  if (pipe_plan(S, a.Hq, a.Hkv, D, dtype, a.c.shift, a.r.total, a.r.max_q, &p)) {
    a.width = p.width;
    a.cuts = reinterpret_cast<int4*>(reinterpret_cast<char*>(a.part) + p.cuts);
    if (dtype == SEKA_F32) return launch_chunk_block_f32(a, D, p, s);
    return D == 128 ? launch_chunk_pipe_d128(a, p, s) : launch_chunk_pipe_d64(a, p, s);
  }
  const RowPlan r = row_plan(a.r.B, S, a.Hq, a.Hkv, D, dtype, a.r.total, a.r.max_q);
  a.p = r.p;
  a.items_of = reinterpret_cast<int4*>(reinterpret_cast<char*>(a.part) + row_states(r, a.Hkv, D));
  return dtype == SEKA_BF16 ? launch_chunk_bf16(a, D, r, s) : launch_chunk_f32(a, D, r, s);
}

}  // namespace seka
