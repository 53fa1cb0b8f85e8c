// New tokens' keys and values to their places in a paged cache, keys and queries turned to their positions on the way.
//
//   token i of member b lies at j = k_len - q_len + i:  K[table[b][j / page], :, j % page] = R((start + j) f) k_i,
//   V[..] = v_i, q_out_i = R((start + j) f) q_i
// HBM-bound: every element is read once and written once.  A warp has one token, or a part of its rows where tokens are few; its rows
// are the query heads, the key heads and the value heads.  A row is spread over d / 16 lanes with two 16-byte pieces each, as in
// the rotation by token index; rows are asked for before the token's angles are made (fp64 up to their remainder), and before the
// lengths are known: of a token behind its member's q_len the first batch of rows is read for nothing.
//
// Measured (us; two prompts of 8192 tokens, 16 + 4 heads of 128, bf16, pages of 64): 35.4, 5.7 TB/s, 88 % of the copy rate (34.0 where nothing
// turns); the rest is the start and end of the kernel and of its waves of CTAs.  Rows asked for behind the lengths and the page 37.1; batches
// ahead and CTAs an SM 4 and 3: 36.4, 4 and 2: 40.5, 6 and 2: 38.8, 2 and 4: 35.4.  64 single tokens: 4.2 on the device.
// Eight prompts padded to 8192 tokens, with q_len: 121.6 if all are full, 68.7 if they have 512 to 8192 (34 % of the tokens; 42 without the
// padding); with the lengths read ahead of the rows, 139.3 and 62.0, and two at 75 % on average 32.2 instead of 29.4.  The lines cross where
// about half the tokens are padding, so the rows come first.
#include "paged.cuh"
#include "rotary.cuh"

namespace mosaic {

namespace {

constexpr int kAppendThreads = 256, kAppendWarps = kAppendThreads / 32;
constexpr int kRounds = 3;  // batches of rows that a warp has on their way

struct AppendArgs {
  View q, q_out, k, v, k_pages, v_pages;
  const double* freqs;
  long long start;
  unsigned tokens;
  int N, d, rot, lanes, heads, kv_heads, parts;
  float amplitude;
};

enum { kStill = 0, kPairs = 1, kHalves = 2 };

// PART: some channels do not turn
template <bool F16, int MODE, bool PART>
__global__ void __launch_bounds__(kAppendThreads, 3) append_kernel(const PagedGeo g, const __grid_constant__ AppendArgs a) {
  constexpr int T = F16 ? kF16 : kBf16, V = Vec<T>::n;
  constexpr bool HALF = MODE == kHalves;
  __shared__ alignas(16) Angles angles[kAppendWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Place pl = place<T, HALF>(a, lane);
  const int zero = await_stream();
  // (the token holds the wait's zero, and with it every address that follows from it: lengths, table, rows)
  const unsigned task = blockIdx.x * kAppendWarps + warp + (unsigned)zero, token = task / (unsigned)a.parts;
  if (token >= a.tokens) return;
  const int part = (int)(task - token * a.parts), b = (int)(token / (unsigned)a.N), n = (int)(token - (unsigned)b * a.N);
  const int rows = a.heads + 2 * a.kv_heads, end = (int)((long long)rows * (part + 1) / a.parts);
  const int ca = 2 * pl.ca, cb = 2 * pl.cb;
  const char* xq = a.q.data + b * a.q.sb + n * a.q.sn;
  const char* xk = a.k.data + b * a.k.sb + n * a.k.sn - a.heads * a.k.sh;
  const char* xv = a.v.data + b * a.v.sb + n * a.v.sn - (a.heads + a.kv_heads) * a.v.sh;
  uint4 va[kRounds], vb[kRounds];
  auto ask = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const int r = r0 + u * pl.groups + pl.group;
      if (r < end) {
        const char* x = r < a.heads ? xq + r * a.q.sh : r < a.heads + a.kv_heads ? xk + r * a.k.sh : xv + r * a.v.sh;
        va[u] = *reinterpret_cast<const uint4*>(x + ca);
        vb[u] = *reinterpret_cast<const uint4*>(x + cb);
      }
    }
  };
  int r0 = (int)((long long)rows * part / a.parts);
  ask(r0);  // (ahead of the lengths and the table, which come one after the other)
  const Span s = span_of(g, b);
  if (n >= s.ql) return;
  const int j = s.off + n;
  int page = j < 0 ? -1 : __ldg(g.table + b * g.table_stride + (j >> g.shift));
  if constexpr (MODE != kStill) {
    still_angles(a, angles[warp], lane);
    make_angles(a, a.freqs + zero, a.start + j, angles[warp], lane);
  }
  page = (unsigned)page < (unsigned)g.pages ? page : -1;  // a token without a page is not kept
  const int slot = j & ((1 << g.shift) - 1);
  char* yq = a.q_out.data + b * a.q_out.sb + n * a.q_out.sn;
  char* yk = a.k_pages.data + page * a.k_pages.sb + slot * a.k_pages.sn - a.heads * a.k_pages.sh;
  char* yv = a.v_pages.data + page * a.v_pages.sb + slot * a.v_pages.sn - (a.heads + a.kv_heads) * a.v_pages.sh;
  for (;;) {
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const int r = r0 + u * pl.groups + pl.group;
      if (r >= end) continue;
      if (MODE != kStill && r < a.heads + a.kv_heads) {
        if constexpr (PART) {
          turn_part<T, HALF>(va[u], vb[u], angles[warp], a, pl);
        } else {
          float fa[V], fb[V];
          widen<T>(va[u], fa);
          widen<T>(vb[u], fb);
          turn_all<V, HALF>(fa, fb, angles[warp], a, pl);
          va[u] = narrow<T>(fa);
          vb[u] = narrow<T>(fb);
        }
      }
      if (r >= a.heads && page < 0) continue;
      char* y = r < a.heads ? yq + r * a.q_out.sh : r < a.heads + a.kv_heads ? yk + r * a.k_pages.sh : yv + r * a.v_pages.sh;
      *reinterpret_cast<uint4*>(y + ca) = va[u];
      *reinterpret_cast<uint4*>(y + cb) = vb[u];
    }
    r0 += kRounds * pl.groups;
    if (r0 >= end) break;
    ask(r0);
  }
}

template <bool F16, int MODE, bool PART>
int launch(const HostCtx& c, const PagedGeo& g, AppendArgs a) {
  int sms = 0;
  if (const int rc = launch_setup(nullptr, 0, nullptr, &sms)) return rc;
  // Few tokens: a token's rows go to several warps, until there are sixteen warps an SM or a warp has one batch of rows.
  const int rows = a.heads + 2 * a.kv_heads, groups = 32 / a.lanes;
  a.parts = 1;
  while ((long long)a.tokens * a.parts < 16ll * sms && a.parts * groups < rows) a.parts *= 2;
  const long long blocks = ((long long)a.tokens * a.parts + kAppendWarps - 1) / kAppendWarps;
  return launch_kernel(append_kernel<F16, MODE, PART>, dim3((unsigned)blocks), kAppendThreads, 0, c.stream, true, 0, g, a);
}
template <bool F16>
int launch(const HostCtx& c, const PagedGeo& g, const AppendArgs& a, bool half) {
  if (a.rot == 0) return launch<F16, kStill, false>(c, g, a);
  if (half) return a.rot < a.d ? launch<F16, kHalves, true>(c, g, a) : launch<F16, kHalves, false>(c, g, a);
  return a.rot < a.d ? launch<F16, kPairs, true>(c, g, a) : launch<F16, kPairs, false>(c, g, a);
}

}  // namespace

int launch_paged_append(const HostCtx& c, const PagedGeo& g, const mosaic_paged_params* p, const double* freqs, const AppendTensors& t) {
  AppendArgs a = {};
  a.d = p->d;
  a.rot = p->rot_dim;
  a.lanes = p->d / 16;
  a.amplitude = p->amplitude > 0.f ? p->amplitude : 1.f;
  a.q = t.q; a.q_out = t.q_out; a.k = t.k; a.v = t.v; a.k_pages = t.k_pages; a.v_pages = t.v_pages;
  a.freqs = freqs;
  a.start = p->start;
  a.tokens = (unsigned)((long long)p->B * p->Nq);
  a.N = p->Nq;
  a.heads = t.q.data ? p->H : 0;
  a.kv_heads = p->Hkv;
  const bool half = (p->flags & MOSAIC_FLAG_HALF_PAIRS) != 0;
  return p->flags & MOSAIC_FLAG_FP16 ? launch<true>(c, g, a, half) : launch<false>(c, g, a, half);
}

}  // namespace mosaic
