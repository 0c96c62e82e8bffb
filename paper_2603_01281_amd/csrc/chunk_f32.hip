// seka_attention_chunk, fp32: products and accumulation on v_mfma_f32_16x16x4_f32.
//
// Rows, ranges and merging as in the bf16 kernel (chunk.hip).  Few rows: a wave's step is 16 keys:
//   S^T (16 keys x 16 rows) = K q^T        lane (row l16, group g) gets keys 4 g + i,
//   O^T (D x 16 rows)      += V^T P^T      for which it has the operand, and ends with d = 64 hh + 16 g + 4 i + x.
// K and V go from the pages straight into operand registers with 16-byte loads, those of the wave's next 16 keys as soon as its
// products with these are issued.  A score is shared by several accumulators: short chains of sums, and no product waits for
// the one before it.
#include "chunk_rows.h"

namespace seka {
namespace {

template <int D, int RT, int NW>
__global__ __launch_bounds__(64 * NW, RT == 4 ? 1 : 2) void chunk_rows_f32_kernel(ChunkArgs a) {
  constexpr int NCH = RT == 1 ? 8 : RT == 2 ? 4 : 2;
  constexpr int KI = D / 16, VH = D / 64, DX = D / 16;
  constexpr int BK = 16, OLD = D + 4, R = 16 * RT;
  __shared__ __attribute__((aligned(16))) float sm_o[NW * 16 * OLD];
  __shared__ float sm_ml[NW][16][2];

  ChunkItem it;
  const bool exists = plan_item(a.r, a.c, a.p, blockIdx.x, it);
  row_describe(a, exists, it);
  if (!exists) return;                     // workgroup-uniform
  int k0, k1;
  plan_range(a.p, it, k0, k1);
  const int h = blockIdx.y, G = a.p.G;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
  const int nrows = it.e.n * G, ctx = it.e.len - it.e.n;

  f32x4 qv[RT][KI];                        // d = 16 i + 4 g + e
  int last[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = it.rc * R + 16 * rt + l16;
    const bool ok = row < nrows;
    const int i = ok ? row / G : 0, hd = ok ? row % G : 0;
    last[rt] = ok ? ctx + i : -1;
    const float* qp = static_cast<const float*>(a.Q) + ((size_t)(it.e.row0 + i) * a.Hq + h * G + hd) * D + 4 * g;
#pragma unroll
    for (int x = 0; x < KI; ++x) {
      qv[rt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (ok) qv[rt][x] = *reinterpret_cast<const f32x4*>(qp + 16 * x);
    }
  }
  const int all_see = ctx + it.rc * R / G;

  const size_t row_floats = (size_t)a.Hkv * D;
  const float* Kh = static_cast<const float*>(a.c.K) + (size_t)h * D + 4 * g;
  const float* Vh = static_cast<const float*>(a.c.V) + (size_t)h * D + 4 * l16;
  const int slots = (1 << a.c.shift) - 1;
  PageWindow<BK, NW> win;
  int block = 0, at = 0;
  f32x4 kv[KI], vv[4][VH];
  auto turn_window = [&](int kb) __attribute__((always_inline)) {
    if (block == win.left) {
      win.load(a.c, it.b, kb, k1);
      block = 0;
    }
    at = block * win.per_block;
    ++block;
  };
  auto row_of = [&](int kb, int key) __attribute__((always_inline)) -> size_t {
    const int page = __shfl(win.entry, at + (win.per_block > 1 ? (key - kb) >> a.c.shift : 0));
    return (((size_t)page << a.c.shift) + (key & slots)) * row_floats;
  };
  auto fetch_k = [&](int kb) __attribute__((always_inline)) {
    const float* kp = Kh + row_of(kb, min(kb + l16, k1 - 1));
#pragma unroll
    for (int x = 0; x < KI; ++x) kv[x] = *reinterpret_cast<const f32x4*>(kp + 16 * x);
  };
  auto fetch_v = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* vp = Vh + row_of(kb, min(kb + 4 * g + i, k1 - 1));
#pragma unroll
      for (int hh = 0; hh < VH; ++hh) vv[i][hh] = *reinterpret_cast<const f32x4*>(vp + 64 * hh);
    }
  };

  f32x4 o[RT][DX];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kRowLow;
    l[rt] = 0.f;
#pragma unroll
    for (int x = 0; x < DX; ++x) o[rt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = a.scale * 1.4426950408889634f;
  constexpr int TURN = NW * BK;
  int kb = k0 + wave * BK;
  if (kb < k1) {
    win.load(a.c, it.b, kb, k1);
    turn_window(kb);
    fetch_k(kb);
    fetch_v(kb);
  }
  row_arrived(qv);
  // MORE: with keys behind these.  (A branch in the loop instead, and the waits are for what both of its sides have in flight, the next keys too:
  // 6 requests at one token over 29278, 32 / 32 heads, 598 us, without 553.)
  auto step = [&](auto more_c) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more_c)::value;
    f32x4 t[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      f32x4 acc[NCH];
#pragma unroll
      for (int c = 0; c < NCH; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KI; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[(4 * x + e) % NCH] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[x][e], qv[rt][x][e], acc[(4 * x + e) % NCH], 0, 0, 0);
#pragma unroll
      for (int half = NCH / 2; half; half /= 2)
#pragma unroll
        for (int c = 0; c < half; ++c) acc[c] += acc[c + half];
      t[rt] = acc[0] * c2;
    }
    if constexpr (MORE) {
      turn_window(kb + TURN);
      fetch_k(kb + TURN);
      asm volatile("" ::: "memory");       // on their way before the softmax
    }
    const bool masked = kb + BK - 1 > all_see || kb + BK > k1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = kRowLow;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (masked && kb + 4 * g + i > last[rt]) t[rt][i] = -INFINITY;
        top = fmaxf(top, t[rt][i]);
      }
      top = groups_max(top);
      const bool raise = top > m[rt] + kRowSlack;
      if (__any(raise)) {
        const float f = raise ? __builtin_amdgcn_exp2f(m[rt] - top) : 1.f;
        if (raise) m[rt] = top;
        l[rt] *= f;
#pragma unroll
        for (int x = 0; x < DX; ++x) o[rt][x] *= f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        t[rt][i] = __builtin_amdgcn_exp2f(t[rt][i] - m[rt]);
        l[rt] += t[rt][i];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < DX; ++x)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[i][x / 4][x % 4], t[rt][i], o[rt][x], 0, 0, 0);
    if constexpr (MORE) {
      fetch_v(kb + TURN);
      asm volatile("" ::: "memory");       // and these before the next products
    }
  };
  for (; kb + TURN < k1; kb += TURN) step(std::true_type{});
  if (kb < k1) step(std::false_type{});

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float lt = groups_sum(l[rt]);
    __syncthreads();
    float* mo = sm_o + wave * 16 * OLD;
#pragma unroll
    for (int hh = 0; hh < VH; ++hh)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(mo + l16 * OLD + 64 * hh + 16 * g + 4 * i) =
            f32x4{o[rt][4 * hh][i], o[rt][4 * hh + 1][i], o[rt][4 * hh + 2][i], o[rt][4 * hh + 3][i]};
    if (g == 0) {
      sm_ml[wave][l16][0] = m[rt];
      sm_ml[wave][l16][1] = lt;
    }
    __syncthreads();
    merge_waves<float, D, NW>(a, it, h, it.rc * R + 16 * rt, sm_o, sm_ml);
  }
}

// Long chunks: waves of 32 rows each that share the keys.  Tiles of 32 keys and values pass through LDS, double-buffered, loaded to
// registers a tile ahead and their page numbers two; a tile's operands are read from LDS once per 32 rows.  Matrix instructions bound it: 256
// of 32 cycles per tile and wave (D = 128) beside 32 LDS reads.
template <int D>
__global__ __launch_bounds__(256, 2) void chunk_block_f32_kernel(ChunkArgs a) {
  constexpr int RT = 2, NW = 4, BK = 32, KI = D / 16, VH = D / 64, DX = D / 16, LD = D + 4;
  constexpr int CPR = D / 4, NL = BK * CPR / 256, RPP = 256 / CPR;       // 16-byte pieces per row, loads per thread, rows per pass
  static_assert(NW * 16 * RT == kBlockRows, "rows of the plan");
  __shared__ __attribute__((aligned(16))) float kt_lds[2][BK * LD], vt_lds[2][BK * LD];

  ChunkItem it;
  const bool exists = plan_item(a.r, a.c, a.p, blockIdx.x, it);
  row_describe(a, exists, it);
  if (!exists) return;                     // workgroup-uniform
  int k0, k1;
  plan_range(a.p, it, k0, k1);
  const int h = blockIdx.y, G = a.p.G, tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int nrows = it.e.n * G, ctx = it.e.len - it.e.n, row_first = it.rc * kBlockRows + 32 * wave;

  f32x4 qv[RT][KI];                        // d = 16 x + 4 g + e
  int last[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = row_first + 16 * rt + l16;
    const bool ok = row < nrows;
    const int i = ok ? row / G : 0, hd = ok ? row - i * G : 0;
    last[rt] = ok ? ctx + i : -1;
    const float* qp = static_cast<const float*>(a.Q) + ((size_t)(it.e.row0 + i) * a.Hq + h * G + hd) * D + 4 * g;
#pragma unroll
    for (int x = 0; x < KI; ++x) {
      qv[rt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (ok) qv[rt][x] = *reinterpret_cast<const f32x4*>(qp + 16 * x);
    }
  }
  const int all_see = ctx + row_first / G;                                       // keys up to here are seen by all of the wave's rows,
  const int some_see = row_first < nrows ? ctx + (min(row_first + 32, nrows) - 1) / G : -1;      // behind here by none

  const size_t row_floats = (size_t)a.Hkv * D;
  const int slots = (1 << a.c.shift) - 1, row = tid / CPR, piece = 4 * (tid % CPR);
  const float* Kh = static_cast<const float*>(a.c.K) + (size_t)h * D + piece;
  const float* Vh = static_cast<const float*>(a.c.V) + (size_t)h * D + piece;
  int pages[NL];
  f32x4 kn[NL], vn[NL];
  auto fetch_pages = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NL; ++x) pages[x] = page_of(a.c, it.b, min(kb + row + RPP * x, k1 - 1));
  };
  auto fetch = [&](int kb) __attribute__((always_inline)) {                      // rows behind the last key repeat it
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      const size_t off = (((size_t)pages[x] << a.c.shift) + (min(kb + row + RPP * x, k1 - 1) & slots)) * row_floats;
      kn[x] = *reinterpret_cast<const f32x4*>(Kh + off);
      vn[x] = *reinterpret_cast<const f32x4*>(Vh + off);
    }
  };
  auto place = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      *reinterpret_cast<f32x4*>(&kt_lds[buf][(row + RPP * x) * LD + piece]) = kn[x];
      *reinterpret_cast<f32x4*>(&vt_lds[buf][(row + RPP * x) * LD + piece]) = vn[x];
    }
  };

  f32x4 o[RT][DX];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kRowLow;
    l[rt] = 0.f;
#pragma unroll
    for (int x = 0; x < DX; ++x) o[rt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = a.scale * 1.4426950408889634f;
  if (k0 < k1) {
    fetch_pages(k0);
    fetch(k0);
    row_arrived(qv);
    place(0);
    if (k0 + BK < k1) fetch_pages(k0 + BK);
  }
  __syncthreads();
  int buf = 0;
  for (int kb = k0; kb < k1; kb += BK, buf ^= 1) {
    const bool more = kb + BK < k1;
    if (more) {
      fetch(kb + BK);
      if (kb + 2 * BK < k1) fetch_pages(kb + 2 * BK);
    }
    if (kb <= some_see) {                  // wave-uniform
      const float* Kt = kt_lds[buf];
      const float* Vt = vt_lds[buf];
      const bool masked = kb + BK - 1 > all_see || kb + BK > k1;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x4 acc[RT][2];                  // even and odd products: two chains per tile of rows
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][0] = acc[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < KI; ++x) {
          const f32x4 kf = *reinterpret_cast<const f32x4*>(Kt + (16 * half + l16) * LD + 16 * x + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[rt][e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qv[rt][x][e], acc[rt][e & 1], 0, 0, 0);
        }
        f32x4 t[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          t[rt] = (acc[rt][0] + acc[rt][1]) * c2;
          float top = kRowLow;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (masked && kb + 16 * half + 4 * g + i > last[rt]) t[rt][i] = -INFINITY;
            top = fmaxf(top, t[rt][i]);
          }
          top = groups_max(top);
          const bool raise = top > m[rt] + kRowSlack;
          if (__any(raise)) {
            const float f = raise ? __builtin_amdgcn_exp2f(m[rt] - top) : 1.f;
            if (raise) m[rt] = top;
            l[rt] *= f;
#pragma unroll
            for (int x = 0; x < DX; ++x) o[rt][x] *= f;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            t[rt][i] = __builtin_amdgcn_exp2f(t[rt][i] - m[rt]);
            l[rt] += t[rt][i];
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int hh = 0; hh < VH; ++hh) {
            const f32x4 vf = *reinterpret_cast<const f32x4*>(Vt + (16 * half + 4 * g + i) * LD + 64 * hh + 4 * l16);
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
              for (int rt = 0; rt < RT; ++rt) o[rt][4 * hh + x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[x], t[rt][i], o[rt][4 * hh + x], 0, 0, 0);
          }
      }
    }
    if (more) place(buf ^ 1);              // read by nobody since the barrier before
    __syncthreads();
  }

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float lt = groups_sum(l[rt]);
    const int r = row_first + 16 * rt + l16;
    if (r < nrows) {
#pragma unroll
      for (int hh = 0; hh < VH; ++hh)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = 64 * hh + 16 * g + 4 * i;
          row_emit<float, D>(a, it, h, r, d, m[rt], lt, f32x4{o[rt][4 * hh][i], o[rt][4 * hh + 1][i], o[rt][4 * hh + 2][i], o[rt][4 * hh + 3][i]});
        }
    }
  }
}

template <int D, int NW>
void launch_rows(const ChunkArgs& a, const RowPlan& r, hipStream_t s) {
  const dim3 grid(r.items, a.Hkv), block(64 * NW);
  if (r.rows16 == 1) hipLaunchKernelGGL((chunk_rows_f32_kernel<D, 1, NW>), grid, block, 0, s, a);
  else if (r.rows16 == 2) hipLaunchKernelGGL((chunk_rows_f32_kernel<D, 2, NW>), grid, block, 0, s, a);
  else if constexpr (D == 64) hipLaunchKernelGGL((chunk_rows_f32_kernel<D, 4, 4>), grid, dim3(256), 0, s, a);
}

template <int D>
hipError_t launch_rows(const ChunkArgs& a, const RowPlan& r, hipStream_t s) {
  if (r.block) hipLaunchKernelGGL((chunk_block_f32_kernel<D>), dim3(r.items, a.Hkv), dim3(256), 0, s, a);
  else if (r.waves == 8) launch_rows<D, 8>(a, r, s);
  else launch_rows<D, 4>(a, r, s);
  launch_chunk_merge<float, D>(a, r.items, r.rows, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_f32(const ChunkArgs& a, int D, const RowPlan& r, hipStream_t s) {
  return D == 128 ? launch_rows<128>(a, r, s) : launch_rows<64>(a, r, s);
}

}  // namespace seka
