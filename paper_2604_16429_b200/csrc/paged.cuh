// Geometry of the paged cache shared by the kernels that write and read it.
#pragma once
#include "window.cuh"

namespace mosaic {

constexpr int kMinPage = 16;    // slots of a page at least: a step of the attention never leaves one
constexpr int kMaxNew = 16;     // new tokens a sequence that the attention takes
constexpr int kChunkKeys = 512; // keys whose attention is one part, joined with the others at the end

// A pool of pages and the table that says which of them hold a member's tokens: token j lies in slot j % page of page
// table[b][j / page].
struct PagedGeo {
  int B, H, Hkv, G, T, d;  // T: rows of q a member
  int shift, pages, width; // log2 of a page's slots; pages of the pool; entries of a table row
  int window, sinks;       // window 0: none
  long long table_stride;
  const int32_t *table, *k_len, *q_len;
  float scale_log2;
};

// Lengths of member b: its new tokens are the last ql of its kl
__device__ __forceinline__ Span span_of(const PagedGeo& g, int b) {
  Span s;
  s.ql = g.q_len ? min(max(__ldg(g.q_len + b), 0), g.T) : g.T;
  s.kl = min(max(__ldg(g.k_len + b), 0), g.width << g.shift);
  s.off = s.kl - s.ql;
  return s;
}

// A pool as a tensor [pages, Hkv, page, d], strides in bytes
int check_pool(const mosaic_view* v, const mosaic_paged_params* p, View* out);

struct AppendTensors {
  View q, q_out, k, v, k_pages, v_pages;
};
int launch_paged_append(const HostCtx& c, const PagedGeo& g, const mosaic_paged_params* p, const double* freqs, const AppendTensors& t);

}  // namespace mosaic
