// C ABI of libseka: host-side argument validation and dispatch to the HIP launchers.
// Every check here runs before any GPU work is issued, so error paths need no GPU.
#include <cmath>
#include <cstring>

#include "common.h"
#include "paged.h"

namespace {

thread_local hipError_t g_last_hip_error = hipSuccess;

seka_status launch_status(hipError_t e) {
  g_last_hip_error = e;
  if (e == hipSuccess) return SEKA_OK;
  return e == hipErrorNotSupported ? SEKA_ERR_UNSUPPORTED : SEKA_ERR_LAUNCH;
}

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline size_t elem_size(int dtype) { return dtype == SEKA_BF16 ? 2 : 4; }

// Launch grids put the batch (or batch x KV heads) on the y or z axis, which HIP limits to 65535 workgroups.
constexpr int64_t kMaxGridYZ = 65535;

seka_status check_shape(const seka_shape* sh, bool need_q_heads) {
  if (!sh) return SEKA_ERR_NULL;
  if (sh->dtype != SEKA_F32 && sh->dtype != SEKA_BF16) return SEKA_ERR_DTYPE;
  if (sh->B < 1 || sh->S < 1 || sh->Hkv < 1 || sh->Hkv > SEKA_MAX_KV_HEADS) return SEKA_ERR_SHAPE;
  if (sh->D != 64 && sh->D != 128) return SEKA_ERR_SHAPE;
  if (need_q_heads && (sh->Hq < 1 || sh->Hq % sh->Hkv != 0)) return SEKA_ERR_SHAPE;
  if (!std::isfinite(sh->softmax_scale)) return SEKA_ERR_SHAPE;
  // 32-bit element indexing inside one (batch) slice is assumed by the kernels
  const int64_t heads = need_q_heads ? sh->Hq : sh->Hkv;
  if ((int64_t)sh->S * heads * sh->D >= ((int64_t)1 << 31)) return SEKA_ERR_SHAPE;
  return SEKA_OK;
}

seka_status check_steer(const seka_steer* st, const seka_shape* sh) {
  if (!st->U || !st->gain || !st->mask) return SEKA_ERR_NULL;
  if (st->M < 1 || st->M > SEKA_MAX_EXPERTS || st->r < 1) return SEKA_ERR_SHAPE;
  if ((int64_t)st->M * st->r > SEKA_MAX_RANK) return SEKA_ERR_SHAPE;
  if (st->r > sh->D) return SEKA_ERR_SHAPE;
  if (misaligned(st->U) || (st->w && misaligned(st->w))) return SEKA_ERR_ALIGN;
  for (int h = 0; h < sh->Hkv; ++h) {
    if (!std::isfinite(st->gain[h])) return SEKA_ERR_SHAPE;
    if (st->key_scale && !std::isfinite(st->key_scale[h])) return SEKA_ERR_SHAPE;
  }
  if (sh->dtype == SEKA_BF16 && st->r % 8 != 0) return SEKA_ERR_UNSUPPORTED;
  return SEKA_OK;
}

void fill_steer(seka::SteerArgs& sa, const seka_steer* st, int Hkv) {
  std::memset(&sa, 0, sizeof(sa));
  sa.U = st->U;
  sa.w = st->w;
  sa.mask = st->mask;
  sa.M = st->M;
  sa.r = st->r;
  for (int h = 0; h < Hkv; ++h) {
    sa.gain[h] = st->gain[h];
    sa.kscale[h] = st->key_scale ? st->key_scale[h] : 1.0f;
  }
}

bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// seq_lens: padded batch with per-prompt lengths; cu_seqlens (with total_tokens): packed batch; at most one of them.
seka_status attention_common(const void* Q, const void* K, const void* V, void* O, float* lse,
                             const seka_shape* sh, const seka_steer* st, const int32_t* seq_lens,
                             const int32_t* cu_seqlens, int64_t total_tokens, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if (!Q || !K || !V || !O) return SEKA_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || (lse && misaligned(lse)))
    return SEKA_ERR_ALIGN;
  if (seq_lens && (reinterpret_cast<uintptr_t>(seq_lens) & 3u)) return SEKA_ERR_ALIGN;
  if (cu_seqlens && (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u)) return SEKA_ERR_ALIGN;
  if (cu_seqlens && (total_tokens < 1 || total_tokens > 0x7fffffffLL)) return SEKA_ERR_SHAPE;
  const size_t es = elem_size(sh->dtype);
  const size_t tokens = cu_seqlens ? (size_t)total_tokens : (size_t)sh->B * sh->S;
  const size_t nq = tokens * sh->Hq * sh->D * es;
  const size_t nk = tokens * sh->Hkv * sh->D * es;
  if (ranges_overlap(O, nq, Q, nq) || ranges_overlap(O, nq, K, nk) || ranges_overlap(O, nq, V, nk))
    return SEKA_ERR_ALIAS;

  bool steered = false;
  seka::SteerArgs sa;
  if (st && st->mask) {
    rc = check_steer(st, sh);
    if (rc != SEKA_OK) return rc;
    for (int h = 0; h < sh->Hkv; ++h) steered |= (st->gain[h] != 0.0f);
    if (steered) fill_steer(sa, st, sh->Hkv);
  }

  seka::AttnArgs a;
  a.Q = Q; a.K = K; a.V = V; a.O = O; a.lse = lse; a.lens = seq_lens;
  a.cu = cu_seqlens; a.total = cu_seqlens ? (int)total_tokens : 0;
  a.B = sh->B; a.S = sh->S; a.Hq = sh->Hq; a.Hkv = sh->Hkv; a.D = sh->D;
  a.scale = sh->softmax_scale > 0.0f ? sh->softmax_scale : 1.0f / std::sqrt((float)sh->D);
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  (void)hipGetLastError();   // drop any stale error left by earlier, unrelated runtime calls of this thread
  hipError_t e = (sh->dtype == SEKA_BF16)
                     ? seka::launch_attention_bf16(a, steered ? &sa : nullptr, stream)
                     : seka::launch_attention_f32(a, steered ? &sa : nullptr, stream);
  return launch_status(e);
}

// ---- caches of pages ----
constexpr double kTwoPi = 6.283185307179586476925286766559;

size_t pool_bytes(const seka_paged* c, const seka_shape* sh) {
  return (size_t)c->num_pages * c->page_size * sh->Hkv * sh->D * elem_size(sh->dtype);
}
size_t pool_weight_bytes(const seka_paged* c, const seka_shape* sh) { return (size_t)c->num_pages * c->page_size * sh->Hkv * sizeof(float); }

constexpr int64_t kMaxNewTokens = 1 << 24;       // a workgroup of 256 threads each, in a grid of fewer than 2^32 threads

seka_status check_paged(const seka_paged* c, const seka_shape* sh, bool need_w, bool need_lens) {
  if (!c || !c->K || !c->V || !c->table || (need_lens && !c->lens) || (need_w && !c->W)) return SEKA_ERR_NULL;
  if (c->num_pages < 1 || c->max_pages < 1) return SEKA_ERR_SHAPE;
  if (c->page_size < 8 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return SEKA_ERR_SHAPE;
  if (sh->B > kMaxGridYZ) return SEKA_ERR_SHAPE;
  if (misaligned(c->K) || misaligned(c->V) || (c->W && misaligned(c->W))) return SEKA_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(c->table) & 3u) || (c->lens && (reinterpret_cast<uintptr_t>(c->lens) & 3u))) return SEKA_ERR_ALIGN;
  return SEKA_OK;
}

seka::PagedCache paged(const seka_paged* c, const seka_shape* sh) {
  seka::PagedCache p;
  p.K = c->K; p.V = c->V; p.W = c->W; p.table = c->table; p.lens = c->lens;
  p.num_pages = c->num_pages; p.max_pages = c->max_pages;
  p.shift = 0;
  while ((1 << p.shift) < c->page_size) ++p.shift;
  const int64_t room = (int64_t)c->max_pages * c->page_size;
  p.cap = (int)(room < sh->S ? room : sh->S);
  return p;
}

// New tokens of a call; max_q is what a kernel may take for the longest chunk.
seka_status check_chunk(const int32_t* cu, int64_t total, int32_t max_q, const seka_shape* sh, seka::ChunkRows* r) {
  if (!cu) return SEKA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(cu) & 3u) return SEKA_ERR_ALIGN;
  if (total < 1 || total >= kMaxNewTokens || max_q < 1 || max_q > sh->S) return SEKA_ERR_SHAPE;
  r->cu = cu; r->B = sh->B; r->total = (int)total; r->max_q = max_q;
  return SEKA_OK;
}

seka_status check_rope(const seka_rope* rope, const seka_shape* sh, seka::RotaryArgs* a) {
  if (!rope->freq) return SEKA_ERR_NULL;
  if (rope->dim < 2 || rope->dim > sh->D || rope->dim % 2 || !std::isfinite(rope->factor)) return SEKA_ERR_SHAPE;
  for (int i = 0; i < rope->dim / 2; ++i) {
    if (!std::isfinite(rope->freq[i])) return SEKA_ERR_SHAPE;
    a->turns[i] = rope->freq[i] / kTwoPi;
  }
  a->half = rope->dim / 2;
  a->interleaved = rope->interleaved != 0;
  a->factor = rope->factor == 0.0f ? 1.0f : rope->factor;
  return SEKA_OK;
}

float scale_of(const seka_shape* sh) { return sh->softmax_scale > 0.0f ? sh->softmax_scale : 1.0f / std::sqrt((float)sh->D); }

}  // namespace

extern "C" {

const char* seka_status_string(int32_t status) {
  switch (status) {
    case SEKA_OK: return "ok";
    case SEKA_ERR_NULL: return "a required pointer is NULL";
    case SEKA_ERR_SHAPE: return "a dimension or scalar argument is out of range";
    case SEKA_ERR_DTYPE: return "unknown element type";
    case SEKA_ERR_ALIGN: return "a device pointer is not 16-byte aligned";
    case SEKA_ERR_ALIAS: return "an output overlaps an input";
    case SEKA_ERR_UNSUPPORTED: return "no kernel for this request";
    case SEKA_ERR_LAUNCH: return "HIP reported an error on launch";
    case SEKA_ERR_WORKSPACE: return "workspace missing or too small";
    default: return "unknown status";
  }
}

const char* seka_last_launch_error(void) { return hipGetErrorString(g_last_hip_error); }

size_t seka_route_workspace_bytes(const seka_shape* sh, int32_t t0, int32_t t1) {
  if (check_shape(sh, true) != SEKA_OK || t0 < 0 || t1 <= t0 || t1 > sh->S) return 0;
  return seka::route_workspace_bytes(sh->B, sh->Hkv, sh->D, t0, t1);
}

seka_status seka_route(const void* Q, const seka_shape* sh, const float* proto, int32_t M, int32_t t0,
                       int32_t t1, int32_t mode, float tau, float* w_out, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if (!Q || !proto || !w_out) return SEKA_ERR_NULL;
  if (M < 1 || M > SEKA_MAX_EXPERTS) return SEKA_ERR_SHAPE;
  if (t0 < 0 || t1 <= t0 || t1 > sh->S) return SEKA_ERR_SHAPE;
  if ((int64_t)sh->B * sh->Hkv > kMaxGridYZ) return SEKA_ERR_SHAPE;
  if (mode != SEKA_ROUTE_SOFTMAX_COS && mode != SEKA_ROUTE_PAPER_EQ6) return SEKA_ERR_UNSUPPORTED;
  if (!std::isfinite(tau)) return SEKA_ERR_SHAPE;
  if (misaligned(Q) || misaligned(proto) || (reinterpret_cast<uintptr_t>(w_out) & 3u)) return SEKA_ERR_ALIGN;
  const size_t need = seka::route_workspace_bytes(sh->B, sh->Hkv, sh->D, t0, t1);
  if (!workspace || workspace_bytes < need) return SEKA_ERR_WORKSPACE;
  if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  (void)hipGetLastError();
  hipError_t e = seka::launch_route(Q, sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype, proto, M, t0, t1, mode,
                                    tau, w_out, workspace, reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

size_t seka_route_ragged_workspace_bytes(const seka_shape* sh, int32_t window) {
  if (check_shape(sh, true) != SEKA_OK || window < 1) return 0;
  return seka::route_workspace_bytes(sh->B, sh->Hkv, sh->D, 0, window < sh->S ? window : sh->S);
}

seka_status seka_route_ragged(const void* Q, const seka_shape* sh, const float* proto, int32_t M,
                              const int32_t* seq_lens, const int32_t* cu_seqlens, int64_t total_tokens,
                              int32_t window, int32_t mode, float tau, float* w_out, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if (!Q || !proto || !w_out) return SEKA_ERR_NULL;
  if (!seq_lens && !cu_seqlens) return SEKA_ERR_NULL;
  if (M < 1 || M > SEKA_MAX_EXPERTS || window < 1) return SEKA_ERR_SHAPE;
  if ((int64_t)sh->B * sh->Hkv > kMaxGridYZ) return SEKA_ERR_SHAPE;
  if (cu_seqlens && (total_tokens < 1 || total_tokens > 0x7fffffffLL)) return SEKA_ERR_SHAPE;
  if (mode != SEKA_ROUTE_SOFTMAX_COS && mode != SEKA_ROUTE_PAPER_EQ6) return SEKA_ERR_UNSUPPORTED;
  if (!std::isfinite(tau)) return SEKA_ERR_SHAPE;
  if (misaligned(Q) || misaligned(proto) || (reinterpret_cast<uintptr_t>(w_out) & 3u)) return SEKA_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(seq_lens) & 3u) || (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u)) return SEKA_ERR_ALIGN;
  const int win = window < sh->S ? window : sh->S;
  const size_t need = seka::route_workspace_bytes(sh->B, sh->Hkv, sh->D, 0, win);
  if (!workspace || workspace_bytes < need) return SEKA_ERR_WORKSPACE;
  if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  (void)hipGetLastError();
  hipError_t e = seka::launch_route(Q, sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype, proto, M, 0, win, mode, tau,
                                    w_out, workspace, reinterpret_cast<hipStream_t>(hip_stream),
                                    cu_seqlens ? nullptr : seq_lens, cu_seqlens, cu_seqlens ? (int)total_tokens : 0, win);
  return launch_status(e);
}

size_t seka_project_route_workspace_bytes(const seka_shape* sh) {
  if (check_shape(sh, true) != SEKA_OK || sh->D != 128 || sh->S % 128 != 0) return 0;
  return seka::project_route_workspace_bytes(sh->B, sh->S, sh->Hq);
}

seka_status seka_project_route(const void* X, const void* Wq, int32_t E, void* Q_out, const seka_shape* sh,
                               const float* proto, int32_t M, int32_t mode, float tau, float* w_out,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if (!X || !Wq || !Q_out) return SEKA_ERR_NULL;
  if (E < 64 || E % 64 != 0) return SEKA_ERR_SHAPE;
  if ((int64_t)sh->B * sh->S / 128 > kMaxGridYZ || (int64_t)sh->B * sh->Hkv > kMaxGridYZ) return SEKA_ERR_SHAPE;
  if (sh->dtype != SEKA_BF16 || sh->D != 128 || sh->S % 128 != 0) return SEKA_ERR_UNSUPPORTED;
  if ((int64_t)sh->Hq * sh->D * (int64_t)E >= ((int64_t)1 << 40)) return SEKA_ERR_SHAPE;
  if (misaligned(X) || misaligned(Wq) || misaligned(Q_out)) return SEKA_ERR_ALIGN;
  const size_t nx = (size_t)sh->B * sh->S * E * 2, nw = (size_t)sh->Hq * sh->D * E * 2;
  const size_t nq = (size_t)sh->B * sh->S * sh->Hq * sh->D * 2;
  if (ranges_overlap(Q_out, nq, X, nx) || ranges_overlap(Q_out, nq, Wq, nw)) return SEKA_ERR_ALIAS;
  if (w_out) {
    if (!proto) return SEKA_ERR_NULL;
    if (M < 1 || M > SEKA_MAX_EXPERTS) return SEKA_ERR_SHAPE;
    if (mode != SEKA_ROUTE_SOFTMAX_COS && mode != SEKA_ROUTE_PAPER_EQ6) return SEKA_ERR_UNSUPPORTED;
    if (!std::isfinite(tau)) return SEKA_ERR_SHAPE;
    if (misaligned(proto) || (reinterpret_cast<uintptr_t>(w_out) & 3u)) return SEKA_ERR_ALIGN;
    const size_t need = seka::project_route_workspace_bytes(sh->B, sh->S, sh->Hq);
    if (!workspace || workspace_bytes < need) return SEKA_ERR_WORKSPACE;
    if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  }
  (void)hipGetLastError();
  hipError_t e = seka::launch_project_route(X, Wq, E, Q_out, sh->B, sh->S, sh->Hq, sh->Hkv, proto, M, mode, tau, w_out,
                                            workspace, reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

seka_status seka_edit_keys(const void* K_in, void* K_out, const seka_shape* sh, const seka_steer* st,
                           void* hip_stream) {
  seka_status rc = check_shape(sh, false);
  if (rc != SEKA_OK) return rc;
  if (!K_in || !K_out || !st) return SEKA_ERR_NULL;
  if (sh->B > kMaxGridYZ) return SEKA_ERR_SHAPE;
  rc = check_steer(st, sh);
  if (rc != SEKA_OK) return rc;
  if (misaligned(K_in) || misaligned(K_out)) return SEKA_ERR_ALIGN;
  const size_t nk = (size_t)sh->B * sh->S * sh->Hkv * sh->D * elem_size(sh->dtype);
  if (K_in != K_out && ranges_overlap(K_in, nk, K_out, nk)) return SEKA_ERR_ALIAS;
  seka::SteerArgs sa;
  fill_steer(sa, st, sh->Hkv);
  (void)hipGetLastError();
  hipError_t e = seka::launch_edit_keys(K_in, K_out, sh->B, sh->S, sh->Hkv, sh->D, sh->dtype, sa,
                                        reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

seka_status seka_edit_keys_packed(const void* K_in, void* K_out, const seka_shape* sh, const seka_steer* st,
                                  const int32_t* cu_seqlens, int64_t total_tokens, void* hip_stream) {
  seka_status rc = check_shape(sh, false);
  if (rc != SEKA_OK) return rc;
  if (!K_in || !K_out || !st || !cu_seqlens) return SEKA_ERR_NULL;
  if (sh->B > kMaxGridYZ) return SEKA_ERR_SHAPE;
  rc = check_steer(st, sh);
  if (rc != SEKA_OK) return rc;
  if (total_tokens < 1 || total_tokens > 0x7fffffffLL) return SEKA_ERR_SHAPE;
  if (misaligned(K_in) || misaligned(K_out) || (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u)) return SEKA_ERR_ALIGN;
  const size_t nk = (size_t)total_tokens * sh->Hkv * sh->D * elem_size(sh->dtype);
  if (K_in != K_out && ranges_overlap(K_in, nk, K_out, nk)) return SEKA_ERR_ALIAS;
  seka::SteerArgs sa;
  fill_steer(sa, st, sh->Hkv);
  (void)hipGetLastError();
  hipError_t e = seka::launch_edit_keys(K_in, K_out, sh->B, sh->S, sh->Hkv, sh->D, sh->dtype, sa,
                                        reinterpret_cast<hipStream_t>(hip_stream), cu_seqlens, (int)total_tokens);
  return launch_status(e);
}

size_t seka_decode_workspace_bytes(const seka_shape* sh) {
  if (check_shape(sh, true) != SEKA_OK) return 0;
  return seka::decode_workspace_bytes(sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype);
}

namespace {
// Validation shared by the two generation-step entry points; *need = bytes of partial states the launch cannot do without.
seka_status check_decode(const void* q, const void* K, const void* V, void* O, float* lse, const int32_t* seq_lens,
                         const seka_shape* sh, size_t* need) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if (!q || !K || !V || !O) return SEKA_ERR_NULL;
  if (sh->B > kMaxGridYZ) return SEKA_ERR_SHAPE;
  if (misaligned(q) || misaligned(K) || misaligned(V) || misaligned(O)) return SEKA_ERR_ALIGN;
  if ((lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) || (seq_lens && (reinterpret_cast<uintptr_t>(seq_lens) & 3u)))
    return SEKA_ERR_ALIGN;
  const size_t es = elem_size(sh->dtype);
  const size_t nq = (size_t)sh->B * sh->Hq * sh->D * es;
  const size_t nk = (size_t)sh->B * sh->S * sh->Hkv * sh->D * es;
  if (ranges_overlap(O, nq, q, nq) || ranges_overlap(O, nq, K, nk) || ranges_overlap(O, nq, V, nk)) return SEKA_ERR_ALIAS;
  *need = seka::decode_least_bytes(sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype);
  return SEKA_OK;
}
}  // namespace

seka_status seka_attention_decode(const void* q, const void* K, const void* V, void* O, float* lse,
                                  const int32_t* seq_lens, const seka_shape* sh, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  size_t need = 0;
  seka_status rc = check_decode(q, K, V, O, lse, seq_lens, sh, &need);
  if (rc != SEKA_OK) return rc;
  if (!workspace || workspace_bytes < need) return SEKA_ERR_WORKSPACE;
  if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  const float scale = sh->softmax_scale > 0.0f ? sh->softmax_scale : 1.0f / std::sqrt((float)sh->D);
  (void)hipGetLastError();
  hipError_t e = seka::launch_decode(q, K, V, O, lse, seq_lens, sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype, scale,
                                     workspace, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

seka_status seka_attention_decode_static(const void* q, const void* K, const void* V, void* O, float* lse,
                                         const int32_t* seq_lens, const seka_shape* sh, void* hip_stream) {
  size_t need = 0;
  seka_status rc = check_decode(q, K, V, O, lse, seq_lens, sh, &need);
  if (rc != SEKA_OK) return rc;
  if (need > (size_t)SEKA_DECODE_STATIC_MAX_BYTES) return SEKA_ERR_WORKSPACE;   // larger problems: seka_attention_decode
  void* scratch_ptr = nullptr;
  (void)hipGetLastError();
  hipError_t e = seka::decode_static_scratch(&scratch_ptr);
  if (e != hipSuccess) return launch_status(e);
  const float scale = sh->softmax_scale > 0.0f ? sh->softmax_scale : 1.0f / std::sqrt((float)sh->D);
  e = seka::launch_decode(q, K, V, O, lse, seq_lens, sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype, scale, scratch_ptr,
                          seka::kDecodeStaticScratchBytes, reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

size_t seka_learn_workspace_bytes(const seka_shape* sh) {
  if (check_shape(sh, false) != SEKA_OK || (int64_t)sh->B * sh->S >= (1 << 24)) return 0;
  return seka::learn_workspace_bytes(sh->Hkv, sh->D, sh->B * sh->S);
}

seka_status seka_learn_projection(const void* h_neutral, const void* h_signal, const seka_shape* sh, float gamma,
                                  float* U_out, float* sigma_out, int32_t* k_out, void* U_packed, int32_t r_pad,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
  seka_status rc = check_shape(sh, false);
  if (rc != SEKA_OK) return rc;
  if ((int64_t)sh->B * sh->S >= (1 << 24)) return SEKA_ERR_SHAPE;
  if (!h_neutral || !h_signal || !U_out || !sigma_out || !k_out) return SEKA_ERR_NULL;
  if (!(gamma > 0.0f && gamma <= 1.0f)) return SEKA_ERR_SHAPE;
  if (U_packed && (r_pad < 1 || r_pad > sh->D)) return SEKA_ERR_SHAPE;
  if (misaligned(h_neutral) || misaligned(h_signal) || misaligned(U_out) || misaligned(sigma_out) ||
      (U_packed && misaligned(U_packed)) || (reinterpret_cast<uintptr_t>(k_out) & 3u))
    return SEKA_ERR_ALIGN;
  const int n = sh->B * sh->S;
  const size_t nh = (size_t)n * sh->Hkv * sh->D * elem_size(sh->dtype);
  const size_t nu = (size_t)sh->Hkv * sh->D * sh->D * sizeof(float), ns = (size_t)sh->Hkv * sh->D * sizeof(float);
  const void* outs[4] = {U_out, sigma_out, k_out, U_packed};
  const size_t out_bytes[4] = {nu, ns, (size_t)sh->Hkv * sizeof(int32_t),
                               U_packed ? (size_t)sh->Hkv * sh->D * r_pad * elem_size(sh->dtype) : 0};
  for (int i = 0; i < 4; ++i) {
    if (!out_bytes[i]) continue;
    if (ranges_overlap(outs[i], out_bytes[i], h_neutral, nh) || ranges_overlap(outs[i], out_bytes[i], h_signal, nh))
      return SEKA_ERR_ALIAS;
    for (int j = i + 1; j < 4; ++j)
      if (out_bytes[j] && ranges_overlap(outs[i], out_bytes[i], outs[j], out_bytes[j])) return SEKA_ERR_ALIAS;
  }
  const size_t need = seka::learn_workspace_bytes(sh->Hkv, sh->D, n);
  if (!workspace || workspace_bytes < need) return SEKA_ERR_WORKSPACE;
  if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  (void)hipGetLastError();
  hipError_t e = seka::launch_learn(h_neutral, h_signal, n, sh->Hkv, sh->D, sh->dtype, gamma, U_out, sigma_out, k_out,
                                    U_packed, r_pad, workspace, reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

seka_status seka_head_distance(const void* h_pos, const void* h_neg, const seka_shape* sh, float* D_out,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
  seka_status rc = check_shape(sh, false);
  if (rc != SEKA_OK) return rc;
  if ((int64_t)sh->B * sh->S >= (1 << 24)) return SEKA_ERR_SHAPE;
  if (!h_pos || !h_neg || !D_out) return SEKA_ERR_NULL;
  if (misaligned(h_pos) || misaligned(h_neg) || (reinterpret_cast<uintptr_t>(D_out) & 3u)) return SEKA_ERR_ALIGN;
  const int n = sh->B * sh->S;
  const size_t nh = (size_t)n * sh->Hkv * sh->D * elem_size(sh->dtype);
  if (ranges_overlap(D_out, (size_t)sh->Hkv * sizeof(float), h_pos, nh) ||
      ranges_overlap(D_out, (size_t)sh->Hkv * sizeof(float), h_neg, nh))
    return SEKA_ERR_ALIAS;
  if (!workspace || workspace_bytes < seka::learn_workspace_bytes(sh->Hkv, sh->D, n)) return SEKA_ERR_WORKSPACE;
  if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  (void)hipGetLastError();
  hipError_t e = seka::launch_head_distance(h_pos, h_neg, n, sh->Hkv, sh->D, sh->dtype, D_out, workspace,
                                            reinterpret_cast<hipStream_t>(hip_stream));
  return launch_status(e);
}

seka_status seka_attention_prefill(const void* Q, const void* K, const void* V, void* O, float* lse,
                                   const seka_shape* sh, const seka_steer* st, void* hip_stream) {
  return attention_common(Q, K, V, O, lse, sh, st, nullptr, nullptr, 0, hip_stream);
}

seka_status seka_attention_plain(const void* Q, const void* K, const void* V, void* O, float* lse,
                                 const seka_shape* sh, void* hip_stream) {
  return attention_common(Q, K, V, O, lse, sh, nullptr, nullptr, nullptr, 0, hip_stream);
}

seka_status seka_attention_prefill_ragged(const void* Q, const void* K, const void* V, void* O, float* lse,
                                          const seka_shape* sh, const seka_steer* st, const int32_t* seq_lens,
                                          void* hip_stream) {
  return attention_common(Q, K, V, O, lse, sh, st, seq_lens, nullptr, 0, hip_stream);
}

seka_status seka_attention_prefill_packed(const void* Q, const void* K, const void* V, void* O, float* lse,
                                          const seka_shape* sh, const seka_steer* st, const int32_t* cu_seqlens,
                                          int64_t total_tokens, void* hip_stream) {
  if (!cu_seqlens) return SEKA_ERR_NULL;
  return attention_common(Q, K, V, O, lse, sh, st, nullptr, cu_seqlens, total_tokens, hip_stream);
}

seka_status seka_rope_frequencies(int32_t dim, double base, int32_t scaling, double stretch, double original, double fast,
                                  double slow, double* freq_out) {
  if (!freq_out) return SEKA_ERR_NULL;
  if (dim < 2 || dim % 2 || dim > 128 || !std::isfinite(base) || !(base > 1.0)) return SEKA_ERR_SHAPE;
  if (scaling < SEKA_ROPE_PLAIN || scaling > SEKA_ROPE_TURNS) return SEKA_ERR_UNSUPPORTED;
  if (scaling != SEKA_ROPE_PLAIN && (!std::isfinite(stretch) || !(stretch >= 1.0))) return SEKA_ERR_SHAPE;
  const bool parts = scaling == SEKA_ROPE_PARTS || scaling == SEKA_ROPE_TURNS;
  if (parts && !(std::isfinite(original) && original > 0.0 && std::isfinite(fast) && slow > 0.0 && fast > slow)) return SEKA_ERR_SHAPE;
  if (scaling == SEKA_ROPE_BASE && dim == 2) return SEKA_ERR_SHAPE;      // its only pair has frequency 1 whatever the base
  if (scaling == SEKA_ROPE_BASE) base *= std::pow(stretch, (double)dim / (dim - 2));
  const auto pair_of = [&](double turns) { return dim * std::log(original / (kTwoPi * turns)) / (2.0 * std::log(base)); };
  const double lo = parts ? std::fmax(std::floor(pair_of(fast)), 0.0) : 0.0;
  const double hi = parts ? std::fmin(std::ceil(pair_of(slow)), (double)dim - 1) : 0.0;
  for (int i = 0; i < dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / dim);
    double stretched = 0.0;                // share of f / stretch
    if (scaling == SEKA_ROPE_LINEAR) stretched = 1.0;
    if (scaling == SEKA_ROPE_PARTS) stretched = (i - lo) / std::fmax(hi - lo, 1e-3);
    if (scaling == SEKA_ROPE_TURNS) stretched = (fast - original * f / kTwoPi) / (fast - slow);
    stretched = std::fmin(std::fmax(stretched, 0.0), 1.0);
    freq_out[i] = f * (1.0 - stretched) + f / (scaling == SEKA_ROPE_PLAIN ? 1.0 : stretch) * stretched;
  }
  return SEKA_OK;
}

seka_status seka_rotary(const void* Q, void* Q_out, const void* K, void* K_out, const seka_shape* sh, const seka_rope* rope,
                        const int32_t* positions, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if (!Q || !Q_out || !rope || (K == nullptr) != (K_out == nullptr)) return SEKA_ERR_NULL;
  seka::RotaryArgs a = {};
  if ((rc = check_rope(rope, sh, &a)) != SEKA_OK) return rc;
  const int64_t total = (int64_t)sh->B * sh->S;
  if (total >= kMaxNewTokens) return SEKA_ERR_SHAPE;
  if (misaligned(Q) || misaligned(Q_out) || misaligned(K) || misaligned(K_out) || (reinterpret_cast<uintptr_t>(positions) & 3u)) return SEKA_ERR_ALIGN;
  const size_t nq = (size_t)total * sh->Hq * sh->D * elem_size(sh->dtype), nk = K ? (size_t)total * sh->Hkv * sh->D * elem_size(sh->dtype) : 0;
  if ((Q_out != Q && ranges_overlap(Q_out, nq, Q, nq)) ||
      (K && ((K_out != K && ranges_overlap(K_out, nk, K, nk)) || ranges_overlap(Q_out, nq, K, nk) || ranges_overlap(K_out, nk, Q, nq) ||
             ranges_overlap(Q_out, nq, K_out, nk))))
    return SEKA_ERR_ALIAS;
  if (positions && (ranges_overlap(Q_out, nq, positions, (size_t)total * 4) || (K && ranges_overlap(K_out, nk, positions, (size_t)total * 4)))) return SEKA_ERR_ALIAS;
  a.Q = Q; a.Q_out = Q_out; a.K = K; a.K_out = K_out; a.positions = positions;
  a.total = (int)total; a.S = sh->S; a.Hq = sh->Hq; a.Hkv = sh->Hkv; a.D = sh->D;
  (void)hipGetLastError();
  return launch_status(seka::launch_rotary(a, sh->dtype, reinterpret_cast<hipStream_t>(hip_stream)));
}

seka_status seka_cache_append(const void* K, const void* V, const void* Q, void* Q_out, const seka_shape* sh,
                              const seka_paged* cache, const seka_rope* rope, const int32_t* positions, const uint8_t* mask,
                              const int32_t* cu_seqlens, int64_t total_tokens, int32_t max_q, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if ((rc = check_paged(cache, sh, false, true)) != SEKA_OK) return rc;
  if (!K || !V || (Q == nullptr) != (Q_out == nullptr)) return SEKA_ERR_NULL;
  seka::RotaryArgs a = {};
  if ((rc = check_chunk(cu_seqlens, total_tokens, max_q, sh, &a.r)) != SEKA_OK) return rc;
  if (rope) {
    if ((rc = check_rope(rope, sh, &a)) != SEKA_OK) return rc;
  } else if (Q) {
    return SEKA_ERR_UNSUPPORTED;           // nothing to do to the queries
  }
  if (misaligned(K) || misaligned(V) || misaligned(Q) || misaligned(Q_out) || (reinterpret_cast<uintptr_t>(positions) & 3u)) return SEKA_ERR_ALIGN;
  const size_t es = elem_size(sh->dtype), pool = pool_bytes(cache, sh);
  const size_t nq = Q ? (size_t)total_tokens * sh->Hq * sh->D * es : 0, nk = (size_t)total_tokens * sh->Hkv * sh->D * es;
  const void* outs[4] = {cache->K, cache->V, cache->W, Q_out};
  const size_t out_bytes[4] = {pool, pool, cache->W ? pool_weight_bytes(cache, sh) : 0, nq};
  const size_t entries = (size_t)sh->B * cache->max_pages * 4;
  const void* ins[7] = {K, V, Q, positions, mask, cache->table, cache->lens};
  const size_t in_bytes[7] = {nk, nk, nq, positions ? (size_t)total_tokens * 4 : 0, mask ? (size_t)total_tokens : 0, entries, (size_t)sh->B * 4};
  for (int i = 0; i < 4; ++i) {
    if (!out_bytes[i]) continue;
    for (int j = 0; j < 7; ++j)
      if (in_bytes[j] && !(i == 3 && j == 2 && Q_out == Q) && ranges_overlap(outs[i], out_bytes[i], ins[j], in_bytes[j])) return SEKA_ERR_ALIAS;
    for (int j = i + 1; j < 4; ++j)
      if (out_bytes[j] && ranges_overlap(outs[i], out_bytes[i], outs[j], out_bytes[j])) return SEKA_ERR_ALIAS;
  }
  a.Q = Q; a.Q_out = Q_out; a.K = K; a.V = V; a.positions = positions; a.mask = mask;
  a.c = paged(cache, sh);
  a.total = (int)total_tokens; a.S = sh->S; a.Hq = sh->Hq; a.Hkv = sh->Hkv; a.D = sh->D;
  (void)hipGetLastError();
  return launch_status(seka::launch_rotary(a, sh->dtype, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t seka_chunk_workspace_bytes(const seka_shape* sh, int64_t total_tokens, int32_t max_q) {
  if (check_shape(sh, true) != SEKA_OK || sh->B > kMaxGridYZ || total_tokens < 1 || total_tokens >= kMaxNewTokens || max_q < 1 || max_q > sh->S) return 0;
  return seka::chunk_workspace_bytes(sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype, (int)total_tokens, max_q);
}

seka_status seka_attention_chunk(const void* Q, void* O, float* lse, const seka_shape* sh, const seka_paged* cache,
                                 const int32_t* cu_seqlens, int64_t total_tokens, int32_t max_q, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if ((rc = check_paged(cache, sh, false, true)) != SEKA_OK) return rc;
  if (!Q || !O) return SEKA_ERR_NULL;
  seka::ChunkArgs a = {};
  if ((rc = check_chunk(cu_seqlens, total_tokens, max_q, sh, &a.r)) != SEKA_OK) return rc;
  if (misaligned(Q) || misaligned(O) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return SEKA_ERR_ALIGN;
  const size_t nq = (size_t)total_tokens * sh->Hq * sh->D * elem_size(sh->dtype), pool = pool_bytes(cache, sh);
  const size_t nl = lse ? (size_t)total_tokens * sh->Hq * sizeof(float) : 0;
  if (ranges_overlap(O, nq, Q, nq) || ranges_overlap(O, nq, cache->K, pool) || ranges_overlap(O, nq, cache->V, pool)) return SEKA_ERR_ALIAS;
  if (lse && (ranges_overlap(lse, nl, O, nq) || ranges_overlap(lse, nl, Q, nq) || ranges_overlap(lse, nl, cache->K, pool) || ranges_overlap(lse, nl, cache->V, pool)))
    return SEKA_ERR_ALIAS;
  const size_t need = seka::chunk_workspace_bytes(sh->B, sh->S, sh->Hq, sh->Hkv, sh->D, sh->dtype, (int)total_tokens, max_q);
  if (need && (!workspace || workspace_bytes < need)) return SEKA_ERR_WORKSPACE;
  if (misaligned(workspace)) return SEKA_ERR_ALIGN;
  a.Q = Q; a.O = O; a.lse = lse; a.c = paged(cache, sh);
  a.part = static_cast<float*>(workspace);
  a.Hq = sh->Hq; a.Hkv = sh->Hkv; a.scale = scale_of(sh);
  (void)hipGetLastError();
  return launch_status(seka::launch_chunk(a, sh->D, sh->dtype, sh->S, reinterpret_cast<hipStream_t>(hip_stream)));
}

seka_status seka_attention_weights(const void* Q, const float* lse, const seka_shape* sh, const seka_paged* cache,
                                   const float* W_in, const int32_t* cu_seqlens, int64_t total_tokens, int32_t max_q,
                                   int32_t window, float decay, void* hip_stream) {
  seka_status rc = check_shape(sh, true);
  if (rc != SEKA_OK) return rc;
  if ((rc = check_paged(cache, sh, true, true)) != SEKA_OK) return rc;
  if (!Q || !lse) return SEKA_ERR_NULL;
  seka::WeightsArgs a = {};
  if ((rc = check_chunk(cu_seqlens, total_tokens, max_q, sh, &a.r)) != SEKA_OK) return rc;
  if (window < 1 || !std::isfinite(decay)) return SEKA_ERR_SHAPE;
  if (misaligned(Q) || (reinterpret_cast<uintptr_t>(lse) & 3u) || misaligned(W_in)) return SEKA_ERR_ALIGN;
  const size_t nw = pool_weight_bytes(cache, sh), pool = pool_bytes(cache, sh);
  const size_t nq = (size_t)total_tokens * sh->Hq * sh->D * elem_size(sh->dtype), nl = (size_t)total_tokens * sh->Hq * sizeof(float);
  if (ranges_overlap(cache->W, nw, Q, nq) || ranges_overlap(cache->W, nw, lse, nl) || ranges_overlap(cache->W, nw, cache->K, pool) ||
      (W_in && W_in != cache->W && ranges_overlap(cache->W, nw, W_in, nw)))
    return SEKA_ERR_ALIAS;
  a.Q = Q; a.lse = lse; a.W_in = decay != 0.0f ? W_in : nullptr; a.c = paged(cache, sh);
  a.Hq = sh->Hq; a.Hkv = sh->Hkv; a.window = window; a.scale = scale_of(sh); a.decay = decay;
  (void)hipGetLastError();
  return launch_status(seka::launch_weights(a, sh->D, sh->dtype, reinterpret_cast<hipStream_t>(hip_stream)));
}

seka_status seka_cache_evict(const seka_shape* sh, const seka_paged* src, const seka_paged* dst, int32_t budget, int32_t recent,
                             int32_t* kept, int32_t* lens_out, void* hip_stream) {
  seka_status rc = check_shape(sh, false);
  if (rc != SEKA_OK) return rc;
  if ((rc = check_paged(src, sh, true, true)) != SEKA_OK) return rc;
  if ((rc = check_paged(dst, sh, true, false)) != SEKA_OK) return rc;
  if (!kept || !lens_out) return SEKA_ERR_NULL;
  if (budget < 1 || recent < 0 || recent > budget) return SEKA_ERR_SHAPE;
  if ((int64_t)dst->max_pages * dst->page_size < (budget < sh->S ? budget : sh->S)) return SEKA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(kept) & 3u) || (reinterpret_cast<uintptr_t>(lens_out) & 3u)) return SEKA_ERR_ALIGN;
  // a tensor of dst is the same tensor of src or overlaps nothing of it
  const bool same = dst->K == src->K || dst->V == src->V || dst->W == src->W;
  if (same && (dst->K != src->K || dst->V != src->V || dst->W != src->W || dst->num_pages != src->num_pages || dst->page_size != src->page_size))
    return SEKA_ERR_ALIAS;
  const void* t[8] = {src->K, src->V, src->W, dst->K, dst->V, dst->W, kept, lens_out};
  const size_t n[8] = {pool_bytes(src, sh), pool_bytes(src, sh), pool_weight_bytes(src, sh), pool_bytes(dst, sh), pool_bytes(dst, sh),
                       pool_weight_bytes(dst, sh), (size_t)sh->B * sh->Hkv * budget * 4, (size_t)sh->B * 4};
  for (int i = 0; i < 8; ++i)
    for (int j = i + 1; j < 8; ++j)
      if (!(same && j == i + 3 && j < 6) && ranges_overlap(t[i], n[i], t[j], n[j])) return SEKA_ERR_ALIAS;
  const void* tables[3] = {src->table, dst->table, src->lens};
  const size_t nt[3] = {(size_t)sh->B * src->max_pages * 4, (size_t)sh->B * dst->max_pages * 4, (size_t)sh->B * 4};
  for (int i = 0; i < 3; ++i)
    for (int j = 3; j < 8; ++j)
      if (ranges_overlap(tables[i], nt[i], t[j], n[j])) return SEKA_ERR_ALIAS;
  seka::EvictArgs a = {};
  a.src = paged(src, sh);
  a.dst = paged(dst, sh);
  a.kept = kept; a.lens_out = lens_out;
  a.B = sh->B; a.Hkv = sh->Hkv; a.row_bytes = sh->D * (int)elem_size(sh->dtype); a.budget = budget; a.recent = recent;
  (void)hipGetLastError();
  return launch_status(seka::launch_evict(a, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
