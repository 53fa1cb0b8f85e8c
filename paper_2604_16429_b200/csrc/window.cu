// C ABI of the sliding-window attention: argument checks, workspace, launches.
#include <math.h>

#include "window.cuh"

namespace mosaic {

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int check(const mosaic_window_params* p, uint32_t more_flags) {
  if (!p || p->B <= 0 || p->H <= 0 || p->Hkv <= 0 || p->H % p->Hkv || p->Nq <= 0 || p->Nk <= 0 || p->window <= 0 || p->sinks < 0)
    return MOSAIC_E_INVALID_ARG;
  if (p->flags & ~(MOSAIC_FLAG_FP16 | more_flags)) return MOSAIC_E_INVALID_ARG;
  if (!(p->scale == p->scale) || isinf(p->scale)) return MOSAIC_E_INVALID_ARG;
  if ((p->d != 64 && p->d != 128) || p->sinks > kMaxSinks) return MOSAIC_E_UNSUPPORTED;
  if (p->Nq > (1 << 29) || p->Nk > (1 << 29) || (long long)p->B * p->H > (1 << 24)) return MOSAIC_E_UNSUPPORTED;
  return MOSAIC_OK;
}

// A tensor that the tensor-map encoder takes: its rows lie at different places.
int check_input(const mosaic_view* v, int B, int heads, int N, View* out) {
  if (const int rc = check_view(v, B, heads, N, 2, out)) return rc;
  return N > 1 && out->sn == 0 ? MOSAIC_E_UNSUPPORTED : MOSAIC_OK;
}

}  // namespace

int make_win_geo(const mosaic_window_params* p, const int32_t* q_len, const int32_t* k_len, WinGeo* g) {
  g->B = p->B; g->H = p->H; g->Hkv = p->Hkv; g->G = p->H / p->Hkv;
  g->Nq = p->Nq; g->Nk = p->Nk; g->d = p->d;
  g->window = p->window < p->Nk ? p->window : p->Nk;
  g->sinks = p->sinks < p->Nk ? p->sinks : p->Nk;
  g->scale = p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->d);
  g->scale_log2 = g->scale * 1.4426950408889634f;
  g->q_len = q_len;
  g->k_len = k_len;
  return aligned(q_len, 4) && aligned(k_len, 4) ? MOSAIC_OK : MOSAIC_E_MISALIGNED;
}

}  // namespace mosaic

using namespace mosaic;

extern "C" {

size_t mosaic_bsa_window_workspace_bytes(const mosaic_window_params* p, int op) {
  WinGeo g;
  if (check(p, 0) || make_win_geo(p, nullptr, nullptr, &g)) return 0;
  return op == MOSAIC_OP_FWD ? kStatusBytes : op == MOSAIC_OP_BWD ? window_bwd_layout(g).total : 0;
}

int mosaic_bsa_window_fwd(const mosaic_window_params* p, const mosaic_view* q, const mosaic_view* k, const mosaic_view* v,
                          const int32_t* q_len, const int32_t* k_len, const mosaic_view* o, float* lse, void* ws,
                          size_t ws_bytes, void* cuda_stream) {
  int rc = check(p, 0);
  if (rc) return rc;
  View vq, vk, vv, vo;
  if ((rc = check_input(q, p->B, p->H, p->Nq, &vq)) || (rc = check_input(k, p->B, p->Hkv, p->Nk, &vk)) ||
      (rc = check_input(v, p->B, p->Hkv, p->Nk, &vv)) || (rc = check_view(o, p->B, p->H, p->Nq, 2, &vo)))
    return rc;
  if (!lse || !ws) return MOSAIC_E_INVALID_ARG;
  if (!aligned(lse, 4) || !aligned(ws, 256)) return MOSAIC_E_MISALIGNED;
  if (ws_bytes < kStatusBytes) return MOSAIC_E_WORKSPACE_TOO_SMALL;
  WinGeo g;
  if ((rc = make_win_geo(p, q_len, k_len, &g))) return rc;
  if ((rc = device_ok())) return rc;
  HostCtx c = {};
  c.stream = (cudaStream_t)cuda_stream;
  c.status = (int*)ws;
  return launch_window_fwd(c, g, (p->flags & MOSAIC_FLAG_FP16) != 0, vq, vk, vv, vo, lse);
}

int mosaic_bsa_window_bwd(const mosaic_window_params* p, const mosaic_view* q, const mosaic_view* k, const mosaic_view* v,
                          const mosaic_view* o, const float* lse, const mosaic_view* d_o, const int32_t* q_len,
                          const int32_t* k_len, const mosaic_view* dq, const mosaic_view* dk, const mosaic_view* dv, void* ws,
                          size_t ws_bytes, void* cuda_stream) {
  int rc = check(p, 0);
  if (rc) return rc;
  WinBwd t;
  if ((rc = check_input(q, p->B, p->H, p->Nq, &t.q)) || (rc = check_input(k, p->B, p->Hkv, p->Nk, &t.k)) ||
      (rc = check_input(v, p->B, p->Hkv, p->Nk, &t.v)) || (rc = check_view(o, p->B, p->H, p->Nq, 2, &t.o)) ||
      (rc = check_input(d_o, p->B, p->H, p->Nq, &t.d_o)) || (rc = check_view(dq, p->B, p->H, p->Nq, 2, &t.dq)) ||
      (rc = check_view(dk, p->B, p->Hkv, p->Nk, 2, &t.dk)) || (rc = check_view(dv, p->B, p->Hkv, p->Nk, 2, &t.dv)))
    return rc;
  if (!lse || !ws) return MOSAIC_E_INVALID_ARG;
  if (!aligned(lse, 4) || !aligned(ws, 256)) return MOSAIC_E_MISALIGNED;
  WinGeo g;
  if ((rc = make_win_geo(p, q_len, k_len, &g))) return rc;
  if (ws_bytes < window_bwd_layout(g).total) return MOSAIC_E_WORKSPACE_TOO_SMALL;
  if ((rc = device_ok())) return rc;
  t.lse = lse;
  HostCtx c = {};
  c.stream = (cudaStream_t)cuda_stream;
  c.status = (int*)ws;
  return launch_window_bwd(c, g, (p->flags & MOSAIC_FLAG_FP16) != 0, t, ws);
}

int mosaic_bsa_window_decode(const mosaic_window_params* p, const mosaic_view* q, const mosaic_view* k, const mosaic_view* v,
                             const int32_t* k_len, const mosaic_view* o, float* lse, void* cuda_stream) {
  int rc = check(p, MOSAIC_FLAG_ROLLING);
  if (rc) return rc;
  const bool rolling = (p->flags & MOSAIC_FLAG_ROLLING) != 0;
  if (p->Nq != 1 || (rolling && (long long)p->window + p->sinks > p->Nk)) return MOSAIC_E_INVALID_ARG;
  View vq, vk, vv, vo;
  if ((rc = check_view(q, p->B, p->H, 1, 2, &vq)) || (rc = check_view(k, p->B, p->Hkv, p->Nk, 2, &vk)) ||
      (rc = check_view(v, p->B, p->Hkv, p->Nk, 2, &vv)) || (rc = check_view(o, p->B, p->H, 1, 2, &vo)))
    return rc;
  if (!lse) return MOSAIC_E_INVALID_ARG;
  if (!aligned(lse, 4)) return MOSAIC_E_MISALIGNED;
  WinGeo g;
  if ((rc = make_win_geo(p, nullptr, k_len, &g))) return rc;
  if ((rc = device_ok())) return rc;
  HostCtx c = {};
  c.stream = (cudaStream_t)cuda_stream;
  return launch_window_decode(c, g, (p->flags & MOSAIC_FLAG_FP16) != 0, rolling ? p->Nk - p->sinks : 0, vq, vk, vv, vo, lse);
}

}  // extern "C"
