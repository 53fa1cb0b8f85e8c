// C ABI of the paged cache: argument checks, workspace, launches.
#include <math.h>

#include <utility>

#include "paged.cuh"

namespace mosaic {

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int log2_of(int n) {
  int s = 0;
  while ((1 << s) < n) ++s;
  return s;
}

// What all calls have in common
int check(const mosaic_paged_params* p, uint32_t flags) {
  if (!p || p->B <= 0 || p->Hkv <= 0 || p->Nq <= 0 || p->pages <= 0 || p->width <= 0 || p->page <= 0 || p->table_stride < 0)
    return MOSAIC_E_INVALID_ARG;
  if (p->flags & ~flags) return MOSAIC_E_INVALID_ARG;
  if (p->d != 64 && p->d != 128) return MOSAIC_E_UNSUPPORTED;
  if (p->page < kMinPage || p->page > kMaxPage || (p->page & (p->page - 1)) || (long long)p->width * p->page > (1 << 30)) return MOSAIC_E_UNSUPPORTED;
  if (p->table_stride > (1ll << 40)) return MOSAIC_E_UNSUPPORTED;
  return MOSAIC_OK;
}

int make_geo(const mosaic_paged_params* p, const int32_t* table, const int32_t* k_len, const int32_t* q_len, PagedGeo* g) {
  *g = {};
  g->G = p->H / p->Hkv;
  g->scale_log2 = (p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->d)) * 1.4426950408889634f;
  g->B = p->B; g->H = p->H; g->Hkv = p->Hkv; g->T = p->Nq; g->d = p->d;
  g->shift = log2_of(p->page); g->pages = p->pages; g->width = p->width;
  g->window = p->window < p->width * p->page ? p->window : 0;  // (one that holds every token is none)
  g->sinks = p->sinks;
  g->table_stride = p->table_stride;
  g->table = table; g->k_len = k_len; g->q_len = q_len;
  if (!table || !k_len) return MOSAIC_E_INVALID_ARG;
  return aligned(table, 4) && aligned(k_len, 4) && aligned(q_len, 4) ? MOSAIC_OK : MOSAIC_E_MISALIGNED;
}

// Most parts that a member's own keys can have: all chunks of its pages, or those that a window and its first rows' ends touch
int most_parts(const mosaic_paged_params* p) {
  const long long all = ((long long)p->width * p->page + kChunkKeys - 1) / kChunkKeys;
  if (!p->window) return (int)all;
  const long long some = ((long long)p->window + p->Nq - 2 + kChunkKeys - 1) / kChunkKeys + 1 + (p->sinks > 0);
  return (int)(some < all ? some : all);
}

// The attention's own
int check_attention(const mosaic_paged_params* p) {
  if (const int rc = check(p, MOSAIC_FLAG_FP16)) return rc;
  if (p->H <= 0 || p->H % p->Hkv || p->window < 0 || p->sinks < 0 || p->prefix_len < 0) return MOSAIC_E_INVALID_ARG;
  if (!(p->scale == p->scale) || isinf(p->scale)) return MOSAIC_E_INVALID_ARG;
  if (p->Nq > kMaxNew || p->sinks > kMaxSinks || (long long)p->B * p->H > (1 << 24)) return MOSAIC_E_UNSUPPORTED;
  if ((long long)p->H / p->Hkv * p->Nq > (1 << 20)) return MOSAIC_E_UNSUPPORTED;
  if (!paged_parts_fit(p->d, p->H / p->Hkv * p->Nq, (long long)p->B * p->Hkv, most_parts(p))) return MOSAIC_E_UNSUPPORTED;
  return MOSAIC_OK;
}

// Behind the status block the parts: sums [part][row][d], then maximum and sum of weights [part][row]
struct Layout {
  size_t o, ml, total;
};
Layout layout(const mosaic_paged_params* p, int parts) {
  const size_t rows = (size_t)p->B * p->H * p->Nq;
  Layout w;
  w.o = kStatusBytes;
  w.ml = w.o + align256((size_t)parts * rows * p->d * sizeof(float));
  w.total = w.ml + align256((size_t)parts * rows * sizeof(float2));
  return w;
}
// The prefix' own
int check_prefix(const mosaic_paged_params* p) {
  if (p->prefix_len <= 0 || p->window || p->sinks) return MOSAIC_E_INVALID_ARG;
  return p->prefix_len > (1 << 30) || (long long)p->B * p->H * p->Nq > (1 << 28) ? MOSAIC_E_UNSUPPORTED : MOSAIC_OK;
}
int shared_parts(const mosaic_paged_params* p, int* chunk) {
  int keys;
  return prefix_parts(p->prefix_len, p->Hkv, (long long)p->B * p->Nq * (p->H / p->Hkv), chunk ? chunk : &keys);
}
// Members that can have one part only get their results from the kernel that makes it.  Behind a prefix that is a launch less, but the
// kernel joins a row's parts one item after the other: taken up to some 40 parts a CTA.  (us on the device, with the join's kernel and
// without: 33 members behind 16 parts 30.6 and 28.0; 8 behind 32 16.7 and 16.5; 64 of 4 key heads behind 37, two items a CTA, 49.4 and 53.7.)
bool is_direct(const mosaic_paged_params* p, int shared) {
  if (most_parts(p) != 1) return false;
  const long long items = (long long)p->B * p->Hkv * paged_row_blocks(p->d, p->H / p->Hkv * p->Nq);
  return (items + kSms - 1) / kSms * shared <= 40;
}

}  // namespace

// Every row has a place of its own: from the smallest stride on, each reaches beyond all that lies within it.  (Any order of the axes, and
// slices of them; only rows that interleave without being a slice of anything are refused beside those that overlap.)
int check_pool(const mosaic_view* v, const mosaic_paged_params* p, View* out) {
  if (const int rc = check_view(v, p->pages, p->Hkv, p->page, 2, out)) return rc;
  struct { long long stride; int n; } axis[3] = {{out->sn, p->page}, {out->sh, p->Hkv}, {out->sb, p->pages}};
  if (axis[0].stride > axis[1].stride) std::swap(axis[0], axis[1]);
  if (axis[1].stride > axis[2].stride) std::swap(axis[1], axis[2]);
  if (axis[0].stride > axis[1].stride) std::swap(axis[0], axis[1]);
  long long within = 2ll * p->d;  // bytes from the first to behind the last of what the strides so far reach
  for (const auto& x : axis) {
    if (x.n == 1) continue;
    if (x.stride < within || x.stride > (1ll << 61) / x.n) return MOSAIC_E_UNSUPPORTED;
    within += (x.n - 1) * x.stride;
  }
  return MOSAIC_OK;
}

namespace {
PartsOut parts_out(const mosaic_paged_params* p, void* ws, int shared, int all) {
  const Layout w = layout(p, all);
  return {(float*)((char*)ws + w.o), (float2*)((char*)ws + w.ml), (long long)p->B * p->H * p->Nq, shared};
}
size_t workspace(const mosaic_paged_params* p, int shared) {
  const int own = is_direct(p, shared) ? 0 : most_parts(p);
  return shared + own ? layout(p, shared + own).total : kStatusBytes;
}
// Tensors, buffers and device of an attention call, whose parameters have been checked
struct Call {
  HostCtx c;
  PagedGeo g;
  View q, o;
  PoolMaps maps;
  bool f16;
};
int make_call(const mosaic_paged_params* p, int shared, const mosaic_view* q, const mosaic_view* k_pages, const mosaic_view* v_pages,
              const int32_t* table, const int32_t* k_len, const int32_t* q_len, const mosaic_view* o, float* lse, void* ws, size_t ws_bytes,
              void* cuda_stream, Call* t) {
  int rc;
  if ((rc = check_view(q, p->B, p->H, p->Nq, 2, &t->q)) || (rc = check_pool(k_pages, p, &t->maps.k_pages)) ||
      (rc = check_pool(v_pages, p, &t->maps.v_pages)) || (rc = check_view(o, p->B, p->H, p->Nq, 2, &t->o)) ||
      (rc = make_geo(p, table, k_len, q_len, &t->g)))
    return rc;
  if (!lse || !ws) return MOSAIC_E_INVALID_ARG;
  if (!aligned(lse, 4) || !aligned(ws, 256)) return MOSAIC_E_MISALIGNED;
  if (ws_bytes < workspace(p, shared)) return MOSAIC_E_WORKSPACE_TOO_SMALL;
  t->c = {};
  t->c.stream = (cudaStream_t)cuda_stream;
  t->c.status = (int*)ws;
  t->f16 = (p->flags & MOSAIC_FLAG_FP16) != 0;
  if ((rc = device_ok())) return rc;
  return t->maps.make(t->g) ? MOSAIC_OK : MOSAIC_E_CUDA;
}
}  // namespace

}  // namespace mosaic

using namespace mosaic;

extern "C" {

int mosaic_bsa_paged_append(const mosaic_paged_params* p, const mosaic_view* k, const mosaic_view* v, const mosaic_view* k_pages,
                            const mosaic_view* v_pages, const int32_t* table, const int32_t* k_len, const int32_t* q_len,
                            const double* freqs, const mosaic_view* q, const mosaic_view* q_out, void* cuda_stream) {
  int rc = check(p, MOSAIC_FLAG_FP16 | MOSAIC_FLAG_HALF_PAIRS);
  if (rc) return rc;
  if (p->rot_dim < 0 || p->rot_dim % 2 || p->rot_dim > p->d || !(p->amplitude >= 0.f) || isinf(p->amplitude)) return MOSAIC_E_INVALID_ARG;
  if ((p->flags & MOSAIC_FLAG_HALF_PAIRS) && p->rot_dim % 16) return MOSAIC_E_UNSUPPORTED;
  if ((q != nullptr) != (q_out != nullptr) || (q && p->H <= 0) || (p->rot_dim && !freqs)) return MOSAIC_E_INVALID_ARG;
  if (p->start > (1ll << 52) || p->start < -(1ll << 52)) return MOSAIC_E_UNSUPPORTED;
  const int heads = q ? p->H : 0;
  if ((long long)p->B * p->Nq > (1 << 30) || (long long)heads + 2ll * p->Hkv > (1 << 16)) return MOSAIC_E_UNSUPPORTED;
  AppendTensors t = {};
  if ((rc = check_view(k, p->B, p->Hkv, p->Nq, 2, &t.k)) || (rc = check_view(v, p->B, p->Hkv, p->Nq, 2, &t.v)) ||
      (rc = check_pool(k_pages, p, &t.k_pages)) || (rc = check_pool(v_pages, p, &t.v_pages)))
    return rc;
  if (q && ((rc = check_view(q, p->B, heads, p->Nq, 2, &t.q)) || (rc = check_view(q_out, p->B, heads, p->Nq, 2, &t.q_out)))) return rc;
  PagedGeo g;
  if ((rc = make_geo(p, table, k_len, q_len, &g))) return rc;
  if (!aligned(freqs, 8)) return MOSAIC_E_MISALIGNED;
  if ((rc = device_ok())) return rc;
  HostCtx c = {};
  c.stream = (cudaStream_t)cuda_stream;
  return launch_paged_append(c, g, p, freqs, t);
}

size_t mosaic_bsa_paged_workspace_bytes(const mosaic_paged_params* p) {
  if (check_attention(p)) return 0;
  if (!p->prefix_len) return workspace(p, 0);
  return check_prefix(p) ? 0 : workspace(p, shared_parts(p, nullptr));
}

int mosaic_bsa_paged_decode(const mosaic_paged_params* p, const mosaic_view* q, const mosaic_view* k_pages, const mosaic_view* v_pages,
                            const int32_t* table, const int32_t* k_len, const int32_t* q_len, const mosaic_view* o, float* lse, void* ws,
                            size_t ws_bytes, void* cuda_stream) {
  int rc = check_attention(p);
  if (rc) return rc;
  if (p->prefix_len) return MOSAIC_E_INVALID_ARG;
  Call t;
  if ((rc = make_call(p, 0, q, k_pages, v_pages, table, k_len, q_len, o, lse, ws, ws_bytes, cuda_stream, &t))) return rc;
  const bool direct = is_direct(p, 0);
  const int most = most_parts(p);
  const PartsOut parts = parts_out(p, ws, 0, most);
  if ((rc = launch_paged_parts(t.c, t.g, t.f16, t.q, t.maps, parts, most, direct, true, t.o, lse)) || direct) return rc;
  return launch_paged_join(t.c, t.g, t.f16, parts, most, t.o, lse);
}

int mosaic_bsa_prefix_decode(const mosaic_paged_params* p, const mosaic_view* q, const mosaic_view* k_pages, const mosaic_view* v_pages,
                             const int32_t* prefix_table, const int32_t* table, const int32_t* k_len, const int32_t* q_len,
                             const mosaic_view* o, float* lse, void* ws, size_t ws_bytes, void* cuda_stream) {
  int rc = check_attention(p);
  if (rc || (rc = check_prefix(p))) return rc;
  if (!prefix_table) return MOSAIC_E_INVALID_ARG;
  if (!aligned(prefix_table, 4)) return MOSAIC_E_MISALIGNED;
  int chunk = 0;
  const int shared = shared_parts(p, &chunk), most = most_parts(p);
  Call t;
  if ((rc = make_call(p, shared, q, k_pages, v_pages, table, k_len, q_len, o, lse, ws, ws_bytes, cuda_stream, &t))) return rc;
  const bool direct = is_direct(p, shared);
  const PartsOut parts = parts_out(p, ws, shared, direct ? shared : shared + most);
  if ((rc = launch_prefix_fwd(t.c, t.g, t.f16, t.q, t.maps, prefix_table, p->prefix_len, chunk, parts))) return rc;
  if ((rc = launch_paged_parts(t.c, t.g, t.f16, t.q, t.maps, parts, most, direct, false, t.o, lse)) || direct) return rc;
  return launch_paged_join(t.c, t.g, t.f16, parts, shared + most, t.o, lse);
}

}  // extern "C"
