// seka_attention_chunk, fp32: products and accumulation on v_mfma_f32_16x16x4_f32.
//
// Rows, ranges and merging as in the bf16 kernel (chunk.hip).  Few rows: a wave's step is 16 keys:
//   S^T (16 keys x 16 rows) = K q^T        lane (row l16, group g) gets keys 4 g + i,
//   O^T (D x 16 rows)      += V^T P^T      for which it has the operand, and ends with d = 64 hh + 16 g + 4 i + x.
// K and V go from the pages straight into operand registers with 16-byte loads, those of the wave's next 16 keys as soon as its
// products with these are issued.  A score is shared by several accumulators: short chains of sums, and no product waits for
// the one before it.  One token of six requests of up to 29278, 32 / 32 heads, D = 128: 2.9 GB in 555 us, 5.2 TB/s, a large copy's rate.
#include "chunk_join.h"
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

// Long chunks (chunk_plan.h): waves of 32 rows each that share the keys.  Tiles of 32 keys and values pass through LDS, double-buffered, loaded to
// registers a tile ahead and their page numbers two; a tile's operands are read from LDS once per 32 rows.  Matrix instructions bound it: 256
// of 32 cycles per tile and wave (D = 128) beside 32 LDS reads.  Where no more than two waves have rows, two waves each take them and half of a tile.
// 2048 new tokens over 8192, 32 / 8 heads, D = 128: 2.1 ms, 115 of 154 TFLOP/s; 802 over 2522: 285 us (cut into ranges per block of rows: 415).
template <int D>
__global__ __launch_bounds__(256, 2) void chunk_block_f32_kernel(ChunkArgs a) {
  constexpr int RT = 2, NW = PipeF32::WAVES, BK = 32, KI = D / 16, VH = D / 64, DX = D / 16, LD = D + 4;
  constexpr int CPR = D / 4, NL = BK * CPR / 256, RPP = 256 / CPR;       // 16-byte pieces per row, loads per thread, rows per pass
  __shared__ __attribute__((aligned(16))) float tiles[4][BK * LD];
  float (*const kt_lds)[BK * LD] = tiles, (*const vt_lds)[BK * LD] = tiles + 2;
  static_assert(NW == 4 && 2 * RT * (DX + 1) * 64 * 4 <= 4 * BK * LD, "states of two waves in the tiles");

  const int h = blockIdx.x % a.Hkv, item = blockIdx.x / a.Hkv, G = a.Hq / a.Hkv, tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  PipePieces<PipeF32> pieces(a.r, a.c, a.width, G, item);
  if (h == 0 && tid == 0) a.cuts[item] = pieces.note();
  pipe_rows_without_keys<float, D>(a, item, h);

  const size_t row_floats = (size_t)a.Hkv * D;
  const int slots = (1 << a.c.shift) - 1, row = tid / CPR, part = 4 * (tid % CPR);
  const float* Kh = static_cast<const float*>(a.c.K) + (size_t)h * D + part;
  const float* Vh = static_cast<const float*>(a.c.V) + (size_t)h * D + part;
  const float c2 = a.scale * 1.4426950408889634f;
  PipePiece piece;
  while (pieces.next(piece)) {             // workgroup-uniform
    const ChunkExtent e = piece.e;
    const int ctx = e.len - e.n, first = max(ctx, 0), base = pipe_first_row(e), wave0 = pipe_first_wave(e, G) + NW * piece.k;
    const bool halves = pieces.p.half(e, piece.k);
    const int rows_of = halves ? wave & 1 : wave;                        // the wave of the block whose rows these are
    const unsigned row_first = 32u * (unsigned)(wave0 + rows_of);
    f32x4 qv[RT][KI];                      // d = 16 x + 4 g + e
    int last[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const unsigned r = row_first + 16 * rt + l16, at = r / (unsigned)G;
      const int pos = base + (int)at;
      const bool ok = pos >= first && pos < e.len;
      last[rt] = ok ? pos : -1;
      const float* qp = static_cast<const float*>(a.Q) + ((size_t)(e.row0 + (ok ? pos - ctx : 0)) * a.Hq + h * G + (ok ? (int)(r - at * G) : 0)) * D + 4 * g;
#pragma unroll
      for (int x = 0; x < KI; ++x) {
        qv[rt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (ok) qv[rt][x] = *reinterpret_cast<const f32x4*>(qp + 16 * x);
      }
    }
    const int pos0 = base + (int)(row_first / (unsigned)G);
    const int all_see = max(pos0, first);                                          // keys up to here are seen by all of the wave's rows,
    const int some_see = pos0 < e.len ? min(base + (int)((row_first + 31) / (unsigned)G), e.len - 1) : -1;         // behind here by none
    const int k0 = 64 * piece.t0;
    const int k1 = min(64 * piece.t1, min(e.len, base + (int)((32u * (unsigned)(wave0 + NW) - 1) / (unsigned)G) + 1));

    int pages[NL];
    f32x4 kn[NL], vn[NL];
    auto fetch_pages = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < NL; ++x) pages[x] = page_of(a.c, piece.b, min(kb + row + RPP * x, k1 - 1));
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
        *reinterpret_cast<f32x4*>(&kt_lds[buf][(row + RPP * x) * LD + part]) = kn[x];
        *reinterpret_cast<f32x4*>(&vt_lds[buf][(row + RPP * x) * LD + part]) = vn[x];
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
    // 16 keys of a tile: half h16 of the one that starts at kb
    auto half_tile = [&](int kb, int h16, int buf) __attribute__((always_inline)) {
      const float* Kt = kt_lds[buf];
      const float* Vt = vt_lds[buf];
      const bool masked = kb + BK - 1 > all_see || kb + BK > k1;
      f32x4 acc[RT][2];                    // even and odd products: two chains per tile of rows
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) acc[rt][0] = acc[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KI; ++x) {
        const f32x4 kf = *reinterpret_cast<const f32x4*>(Kt + (16 * h16 + l16) * LD + 16 * x + 4 * g);
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
          if (masked && kb + 16 * h16 + 4 * g + i > last[rt]) t[rt][i] = -INFINITY;
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
          const f32x4 vf = *reinterpret_cast<const f32x4*>(Vt + (16 * h16 + 4 * g + i) * LD + 64 * hh + 4 * l16);
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) o[rt][4 * hh + x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[x], t[rt][i], o[rt][4 * hh + x], 0, 0, 0);
        }
    };
    fetch_pages(k0);
    fetch(k0);
    row_arrived(qv);
    place(0);
    if (k0 + BK < k1) fetch_pages(k0 + BK);
    __syncthreads();
    int buf = 0;
    for (int kb = k0; kb < k1; kb += BK, buf ^= 1) {
      const bool more = kb + BK < k1;
      if (more) {
        fetch(kb + BK);
        if (kb + 2 * BK < k1) fetch_pages(kb + 2 * BK);
      }
      if (kb <= some_see) {                // wave-uniform
#pragma nounroll
        for (int h16 = halves ? wave >> 1 : 0; h16 < (halves ? (wave >> 1) + 1 : 2); ++h16) half_tile(kb, h16, buf);
      }
      if (more) place(buf ^ 1);            // read by nobody since the barrier before
      __syncthreads();
    }

    float lt[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) lt[rt] = groups_sum(l[rt]);
    if (halves) {                          // waves 2 and 3 hand theirs over, lane by lane
      f32x4* const at = reinterpret_cast<f32x4*>(&tiles[0][0]) + rows_of * RT * (DX + 1) * 64 + lane;
      if (wave >= 2) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
          for (int x = 0; x < DX; ++x) at[(rt * (DX + 1) + x) * 64] = o[rt][x];
          at[(rt * (DX + 1) + DX) * 64] = f32x4{m[rt], lt[rt], 0.f, 0.f};
        }
      }
      __syncthreads();
      if (wave < 2) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const f32x4 ml = at[(rt * (DX + 1) + DX) * 64];
          const float mm = fmaxf(m[rt], ml[0]), f = __builtin_amdgcn_exp2f(m[rt] - mm), f2 = __builtin_amdgcn_exp2f(ml[0] - mm);
          m[rt] = mm;
          lt[rt] = lt[rt] * f + ml[1] * f2;
#pragma unroll
          for (int x = 0; x < DX; ++x) o[rt][x] = o[rt][x] * f + at[(rt * (DX + 1) + x) * 64] * f2;
        }
      }
      __syncthreads();                     // the tiles are free
    }
    if (!halves || wave < 2) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (last[rt] < 0) continue;
        const unsigned r = row_first + 16 * rt + l16;
        const int head = h * G + (int)(r % (unsigned)G);
        const size_t token = (size_t)(e.row0 + last[rt] - ctx);
        float* dst;
        float f = 1.f;
        if (piece.whole) {
          dst = static_cast<float*>(a.O) + (token * a.Hq + head) * D;
          f = 1.f / lt[rt];
          if (a.lse && g == 0) a.lse[(size_t)head * a.r.total + token] = m[rt] * 0.6931471805599453f + logf(lt[rt]);
        } else {
          dst = a.part + (((size_t)pieces.slot(piece) * a.Hkv + h) * PipeF32::ROWS + 32 * rows_of + 16 * rt + l16) * (D + 4);
          if (g == 0) {
            dst[D] = m[rt];
            dst[D + 1] = lt[rt];
          }
        }
#pragma unroll
        for (int hh = 0; hh < VH; ++hh)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(dst + 64 * hh + 16 * g + 4 * i) =
                f32x4{o[rt][4 * hh][i], o[rt][4 * hh + 1][i], o[rt][4 * hh + 2][i], o[rt][4 * hh + 3][i]} * f;
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
  if (r.waves == 8) launch_rows<D, 8>(a, r, s);
  else launch_rows<D, 4>(a, r, s);
  launch_chunk_merge<float, D>(a, r.items, r.rows, s);
  return hipGetLastError();
}

template <int D>
hipError_t launch_block(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) {
  hipLaunchKernelGGL((chunk_block_f32_kernel<D>), dim3((unsigned)(p.width * a.Hkv)), dim3(64 * PipeF32::WAVES), 0, s, a);
  launch_chunk_join<float, PipeF32, D>(a, p, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_block_f32(const ChunkArgs& a, int D, const PipeChunkPlan& p, hipStream_t s) {
  return D == 128 ? launch_block<128>(a, p, s) : launch_block<64>(a, p, s);
}

hipError_t launch_chunk_f32(const ChunkArgs& a, int D, const RowPlan& r, hipStream_t s) {
  return D == 128 ? launch_rows<128>(a, r, s) : launch_rows<64>(a, r, s);
}

}  // namespace seka
