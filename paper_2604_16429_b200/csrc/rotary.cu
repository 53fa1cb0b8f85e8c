// Rotary position embedding of Q and K by token index, and the root-mean-square norm of their heads in the same pass.
//
//   forward   y = R(p f) (x * r * w),  r = 1 / sqrt(mean(x^2) + eps)  (the rotation alone: y = R(p f) x)
//   backward  g = R(-p f) dy;  dw = sum over rows of g * x * r;  dx = r * (g * w - x * r^2 * mean(g * w * x))
//
// HBM-bound: every element is read once (x and dy in the backward) and written once.  A warp has one token and walks its
// heads; a row of d channels is spread over P lanes (the power of two that holds d / 2V), each with two 16-byte pieces of V
// channels: with half pairs the two pieces hold the pairs' two sides, otherwise they lie next to one another.  So a pair never
// leaves its lane, a row's sums are shuffles among P lanes, and 32 / P rows go through a warp at a time, a few fetched ahead.
// The token's rot_dim/2 angles are the same for all its heads: the warp's lanes share them out, take the product with the
// position in half turns and its remainder in fp64 (an angle of 1e6 radians has 2^-33 of error there, 2^-4 in fp32), and leave
// (cos, sin) in shared memory, from where every lane keeps the V that it needs.
#include <math.h>

#include "common.cuh"

namespace mosaic {

namespace {

enum { kBf16 = 0, kF16 = 1, kF32 = 2 };
constexpr int kHeadThreads = 256, kHeadWarps = kHeadThreads / 32;
constexpr int kMaxHeadDim = 256;
constexpr int kAhead = 4;      // rows a lane group has in flight (forward)
constexpr int kAheadBwd = 2;   // the same in the backward, where a row comes with its gradient

struct HeadTensor {
  View x, g;  // input; gradient of the output (backward)
  View y;     // output, or gradient of the input
  const float* w;
  int heads;
};
struct HeadArgs {
  HeadTensor t[2];
  const int64_t* pos;
  const double* freqs;
  float* partial;  // backward: [CTAs, 2, d] sums of the weights' gradients
  long long pos_stride, tokens;  // tokens: of all batch members
  int N, d, rot, lanes, parts;
  float amplitude, eps;
};

template <int T>
struct Vec { static constexpr int n = T == kF32 ? 4 : 8, bytes = T == kF32 ? 4 : 2; };

template <int T>
__device__ __forceinline__ void widen(const uint4& v, float (&f)[Vec<T>::n]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (T == kF32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack16x2(w[i], T == kF16, f[2 * i], f[2 * i + 1]);
  }
}
template <int T>
__device__ __forceinline__ uint4 narrow(const float (&f)[Vec<T>::n]) {
  if constexpr (T == kF32) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  } else {
    return make_uint4(pack16x2(f[0], f[1], T == kF16), pack16x2(f[2], f[3], T == kF16), pack16x2(f[4], f[5], T == kF16),
                      pack16x2(f[6], f[7], T == kF16));
  }
}

// What a lane does in every row: its two pieces' channels, and the warp's share of rows.
struct Place {
  int ca, cb, first_pair;  // first channel of either piece; the pairs first_pair .. first_pair + V - 1 are this lane's
  int group, groups;       // this lane's row of the `groups` rows that a warp takes at a time
  bool on;                 // the lane has channels (d / 2V may be less than P)
};
template <int T, bool HALF>
__device__ __forceinline__ Place place(const HeadArgs& a, int lane) {
  constexpr int V = Vec<T>::n;
  Place p;
  const int slot = lane & (a.lanes - 1), turning = a.rot / (2 * V);
  p.on = slot * 2 * V < a.d;
  p.ca = HALF && slot < turning ? slot * V : slot * 2 * V;
  p.cb = HALF && slot < turning ? a.rot / 2 + slot * V : slot * 2 * V + V;
  p.first_pair = slot * V;
  p.group = lane / a.lanes;
  p.groups = 32 / a.lanes;
  return p;
}

// (cos, sin) of the token's angles, shared out over the warp; pairs that do not turn get (1, 0)
template <int V>
__device__ __forceinline__ void make_angles(const HeadArgs& a, long long pos, float2* cs, const Place& pl, int lane, float (&c)[V],
                                            float (&s)[V]) {
  for (int i = lane; i < a.rot / 2; i += 32) {
    const double turns = (double)pos * (__ldg(a.freqs + i) * 0.31830988618379067154);  // half turns
    const float r = (float)(turns - 2.0 * rint(0.5 * turns));
    float sn, cn;
    sincospif(r, &sn, &cn);
    cs[i] = make_float2(cn * fabsf(a.amplitude), sn * a.amplitude);  // the launcher negates the factor to turn back
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int i = pl.first_pair + j;
    const float2 v = i < a.rot / 2 ? cs[i] : make_float2(1.f, 0.f);
    c[j] = v.x;
    s[j] = v.y;
  }
  __syncwarp();
}

template <int V, bool HALF>
__device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float& x = HALF ? a[j] : j < V / 2 ? a[2 * j] : b[2 * j - V];
    float& y = HALF ? b[j] : j < V / 2 ? a[2 * j + 1] : b[2 * j - V + 1];
    const float t = x * c[j] - y * s[j];
    y = x * s[j] + y * c[j];
    x = t;
  }
}

__device__ __forceinline__ float row_sum(float v, int lanes) {
  for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int V>
__device__ __forceinline__ void load_weights(const float* w, const Place& pl, float (&wa)[V], float (&wb)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    wa[j] = pl.on ? __ldg(w + pl.ca + j) : 0.f;
    wb[j] = pl.on ? __ldg(w + pl.cb + j) : 0.f;
  }
}

// A token's rows of one tensor: `part` of `parts`
__device__ __forceinline__ void rows_of(int heads, int part, int parts, int& r0, int& r1) {
  r0 = (int)((long long)heads * part / parts);
  r1 = (int)((long long)heads * (part + 1) / parts);
}

template <int T, bool HALF, bool NORM>
__global__ void __launch_bounds__(kHeadThreads) head_kernel(const __grid_constant__ HeadArgs a) {
  constexpr int V = Vec<T>::n, SZ = Vec<T>::bytes;
  __shared__ float2 angles[kHeadWarps][kMaxHeadDim / 2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * kHeadWarps + warp + await_stream(), token = task / a.parts;
  if (token >= a.tokens) return;
  const int part = (int)(task - token * a.parts);
  const long long b = token / a.N, n = token - b * a.N;
  const Place pl = place<T, HALF>(a, lane);
  float c[V], s[V];
  make_angles<V>(a, a.rot ? __ldg(a.pos + b * a.pos_stride + n) : 0, angles[warp], pl, lane, c, s);
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    const HeadTensor& t = a.t[i];
    int r0, r1;
    rows_of(t.heads, part, a.parts, r0, r1);
    const char* x = t.x.data + b * t.x.sb + n * t.x.sn;
    char* y = t.y.data + b * t.y.sb + n * t.y.sn;
    float wa[V], wb[V];
    if constexpr (NORM) load_weights<V>(t.w, pl, wa, wb);
    for (int r = r0 + pl.group; r - pl.group < r1; r += pl.groups * kAhead) {  // (the same trips for the whole warp)
      uint4 va[kAhead], vb[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int h = r + k * pl.groups;
        va[k] = vb[k] = make_uint4(0u, 0u, 0u, 0u);
        if (h < r1 && pl.on) {
          va[k] = *reinterpret_cast<const uint4*>(x + h * t.x.sh + pl.ca * SZ);
          vb[k] = *reinterpret_cast<const uint4*>(x + h * t.x.sh + pl.cb * SZ);
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int h = r + k * pl.groups;
        if (h - pl.group >= r1) break;
        float fa[V], fb[V];
        widen<T>(va[k], fa);
        widen<T>(vb[k], fb);
        if constexpr (NORM) {
          float ss = 0.f;
#pragma unroll
          for (int j = 0; j < V; ++j) ss = fmaf(fa[j], fa[j], fmaf(fb[j], fb[j], ss));
          const float rr = rsqrtf(row_sum(ss, a.lanes) / (float)a.d + a.eps);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            fa[j] *= rr * wa[j];
            fb[j] *= rr * wb[j];
          }
        }
        turn<V, HALF>(fa, fb, c, s);
        if (h < r1 && pl.on) {
          *reinterpret_cast<uint4*>(y + h * t.y.sh + pl.ca * SZ) = narrow<T>(fa);
          *reinterpret_cast<uint4*>(y + h * t.y.sh + pl.cb * SZ) = narrow<T>(fb);
        }
      }
    }
  }
}

// Persistent: the sums of the weights' gradients stay in registers over a CTA's tokens (a lane has the same channels in every
// row), and every CTA leaves one row of partial sums.
template <int T, bool HALF>
__global__ void __launch_bounds__(kHeadThreads) head_bwd_kernel(const __grid_constant__ HeadArgs a) {
  constexpr int V = Vec<T>::n, SZ = Vec<T>::bytes;
  __shared__ float2 angles[kHeadWarps][kMaxHeadDim / 2];
  __shared__ float sums[kHeadWarps][kMaxHeadDim];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Place pl = place<T, HALF>(a, lane);
  const long long first = (long long)blockIdx.x * kHeadWarps + warp + await_stream();
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    const HeadTensor& t = a.t[i];
    float wa[V], wb[V], da[V], db[V];
    load_weights<V>(t.w, pl, wa, wb);
#pragma unroll
    for (int j = 0; j < V; ++j) da[j] = db[j] = 0.f;
    for (long long task = first; task < a.tokens * a.parts; task += (long long)gridDim.x * kHeadWarps) {
      const long long token = task / a.parts, b = token / a.N, n = token - b * a.N;
      int r0, r1;
      rows_of(t.heads, (int)(task - token * a.parts), a.parts, r0, r1);
      float c[V], s[V];
      make_angles<V>(a, a.rot ? __ldg(a.pos + b * a.pos_stride + n) : 0, angles[warp], pl, lane, c, s);
      const char *x = t.x.data + b * t.x.sb + n * t.x.sn, *g = t.g.data + b * t.g.sb + n * t.g.sn;
      char* y = t.y.data + b * t.y.sb + n * t.y.sn;
      for (int r = r0 + pl.group; r - pl.group < r1; r += pl.groups * kAheadBwd) {
        uint4 va[kAheadBwd], vb[kAheadBwd], ga[kAheadBwd], gb[kAheadBwd];
#pragma unroll
        for (int k = 0; k < kAheadBwd; ++k) {
          const int h = r + k * pl.groups;
          va[k] = vb[k] = ga[k] = gb[k] = make_uint4(0u, 0u, 0u, 0u);
          if (h < r1 && pl.on) {
            va[k] = *reinterpret_cast<const uint4*>(x + h * t.x.sh + pl.ca * SZ);
            vb[k] = *reinterpret_cast<const uint4*>(x + h * t.x.sh + pl.cb * SZ);
            ga[k] = *reinterpret_cast<const uint4*>(g + h * t.g.sh + pl.ca * SZ);
            gb[k] = *reinterpret_cast<const uint4*>(g + h * t.g.sh + pl.cb * SZ);
          }
        }
#pragma unroll
        for (int k = 0; k < kAheadBwd; ++k) {
          const int h = r + k * pl.groups;
          if (h - pl.group >= r1) break;
          float fa[V], fb[V], ha[V], hb[V];
          widen<T>(va[k], fa);
          widen<T>(vb[k], fb);
          widen<T>(ga[k], ha);
          widen<T>(gb[k], hb);
          turn<V, HALF>(ha, hb, c, s);
          float ss = 0.f, dot = 0.f;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            ss = fmaf(fa[j], fa[j], fmaf(fb[j], fb[j], ss));
            dot = fmaf(ha[j] * wa[j], fa[j], fmaf(hb[j] * wb[j], fb[j], dot));
          }
          const float rr = rsqrtf(row_sum(ss, a.lanes) / (float)a.d + a.eps);
          const float back = row_sum(dot, a.lanes) * rr * rr / (float)a.d;
#pragma unroll
          for (int j = 0; j < V; ++j) {  // (rows that do not exist are zeros: rr is finite or multiplies zeros)
            const float xa = fa[j] * rr, xb = fb[j] * rr;
            if (h < r1) {
              da[j] = fmaf(ha[j], xa, da[j]);
              db[j] = fmaf(hb[j], xb, db[j]);
            }
            fa[j] = rr * (ha[j] * wa[j] - fa[j] * back);
            fb[j] = rr * (hb[j] * wb[j] - fb[j] * back);
          }
          if (h < r1 && pl.on) {
            *reinterpret_cast<uint4*>(y + h * t.y.sh + pl.ca * SZ) = narrow<T>(fa);
            *reinterpret_cast<uint4*>(y + h * t.y.sh + pl.cb * SZ) = narrow<T>(fb);
          }
        }
      }
    }
    // lane groups, then warps, each in a fixed order
#pragma unroll
    for (int j = 0; j < V; ++j) {
      for (int o = a.lanes; o < 32; o <<= 1) {
        da[j] += __shfl_xor_sync(0xffffffffu, da[j], o);
        db[j] += __shfl_xor_sync(0xffffffffu, db[j], o);
      }
      if (pl.group == 0 && pl.on) {
        sums[warp][pl.ca + j] = da[j];
        sums[warp][pl.cb + j] = db[j];
      }
    }
    __syncthreads();
    if ((int)threadIdx.x < a.d) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kHeadWarps; ++w) v += sums[w][threadIdx.x];
      a.partial[((long long)blockIdx.x * 2 + i) * a.d + threadIdx.x] = v;
    }
    __syncthreads();
  }
}

// Sums of the CTAs' partial rows: 32 columns a CTA, 32 threads a column, joined in a fixed order.
__global__ void __launch_bounds__(1024) weight_sum_kernel(const float* __restrict__ partial, int rows, int d, float* __restrict__ dwq,
                                                          float* __restrict__ dwk) {
  __shared__ float part[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
  partial += await_stream();
  float v = 0.f;
  if (col < 2 * d)
    for (int r = y; r < rows; r += 32) v += partial[(long long)r * 2 * d + col];
  part[y][x] = v;
  __syncthreads();
  v = part[x][y];  // a warp per column now
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int c = blockIdx.x * 32 + y;
  if (x == 0 && c < 2 * d) (c < d ? dwq[c] : dwk[c - d]) = v;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int check(const mosaic_rotary_params* p, bool norm) {
  if (!p || p->B <= 0 || p->H <= 0 || p->Hkv <= 0 || p->N <= 0 || p->H % p->Hkv) return MOSAIC_E_INVALID_ARG;
  const uint32_t known = MOSAIC_FLAG_FP16 | MOSAIC_FLAG_FP32 | MOSAIC_FLAG_HALF_PAIRS | (norm ? 0u : MOSAIC_FLAG_INVERSE);
  if ((p->flags & ~known) || ((p->flags & MOSAIC_FLAG_FP16) && (p->flags & MOSAIC_FLAG_FP32))) return MOSAIC_E_INVALID_ARG;
  if (p->rot_dim < 0 || p->rot_dim % 2 || p->rot_dim > p->d || (!norm && p->rot_dim == 0)) return MOSAIC_E_INVALID_ARG;
  if (!(p->amplitude >= 0.f) || isinf(p->amplitude) || (norm && (!(p->eps >= 0.f) || isinf(p->eps)))) return MOSAIC_E_INVALID_ARG;
  if (p->d <= 0 || p->d % 16 || p->d > kMaxHeadDim) return MOSAIC_E_UNSUPPORTED;
  if ((p->flags & MOSAIC_FLAG_HALF_PAIRS) && p->rot_dim % 16) return MOSAIC_E_UNSUPPORTED;
  if ((long long)p->B * p->N > (1ll << 32)) return MOSAIC_E_UNSUPPORTED;
  return MOSAIC_OK;
}

HeadArgs base_args(const mosaic_rotary_params* p, const int64_t* pos, int64_t pos_stride, const double* freqs) {
  HeadArgs a = {};
  a.pos = pos;
  a.freqs = freqs;
  a.pos_stride = pos_stride;
  a.tokens = (long long)p->B * p->N;
  a.N = p->N;
  a.d = p->d;
  a.rot = p->rot_dim;
  const int v = p->flags & MOSAIC_FLAG_FP32 ? 4 : 8;
  for (a.lanes = 1; a.lanes * 2 * v < p->d;) a.lanes *= 2;
  a.amplitude = p->amplitude > 0.f ? p->amplitude : 1.f;
  a.eps = p->eps;
  a.t[0].heads = p->H;
  a.t[1].heads = p->Hkv;
  return a;
}

// Few tokens: a token's heads go to several warps, until there are sixteen warps an SM or a warp has one round of rows.
int split(const HeadArgs& a, int sms) {
  int parts = 1;
  while (a.tokens * parts < 16ll * sms && parts * (32 / a.lanes) < a.t[0].heads) parts *= 2;
  return parts;
}

template <int T, bool HALF>
int launch_head(HeadArgs a, bool norm, cudaStream_t stream) {
  int sms = 0;
  if (const int rc = launch_setup(nullptr, 0, nullptr, &sms)) return rc;
  a.parts = split(a, sms);
  const long long blocks = (a.tokens * a.parts + kHeadWarps - 1) / kHeadWarps;
  if (blocks > 0x7fffffffll) return MOSAIC_E_UNSUPPORTED;
  return launch_kernel(norm ? head_kernel<T, HALF, true> : head_kernel<T, HALF, false>, dim3((unsigned)blocks), kHeadThreads, 0,
                       stream, true, 0, a);
}
int launch_head(const HeadArgs& a, uint32_t flags, bool norm, cudaStream_t stream) {
  const bool half = (flags & MOSAIC_FLAG_HALF_PAIRS) != 0;
  if (flags & MOSAIC_FLAG_FP32) return half ? launch_head<kF32, true>(a, norm, stream) : launch_head<kF32, false>(a, norm, stream);
  if (flags & MOSAIC_FLAG_FP16) return half ? launch_head<kF16, true>(a, norm, stream) : launch_head<kF16, false>(a, norm, stream);
  return half ? launch_head<kBf16, true>(a, norm, stream) : launch_head<kBf16, false>(a, norm, stream);
}

constexpr int kBwdCtas = 4;  // per SM
template <int T, bool HALF>
int launch_head_bwd(HeadArgs a, int ctas, int sms, cudaStream_t stream) {
  a.parts = split(a, sms);
  return launch_kernel(head_bwd_kernel<T, HALF>, dim3((unsigned)ctas), kHeadThreads, 0, stream, true, 0, a);
}
int launch_head_bwd(const HeadArgs& a, uint32_t flags, int ctas, int sms, cudaStream_t stream) {
  const bool half = (flags & MOSAIC_FLAG_HALF_PAIRS) != 0;
  if (flags & MOSAIC_FLAG_FP32)
    return half ? launch_head_bwd<kF32, true>(a, ctas, sms, stream) : launch_head_bwd<kF32, false>(a, ctas, sms, stream);
  if (flags & MOSAIC_FLAG_FP16)
    return half ? launch_head_bwd<kF16, true>(a, ctas, sms, stream) : launch_head_bwd<kF16, false>(a, ctas, sms, stream);
  return half ? launch_head_bwd<kBf16, true>(a, ctas, sms, stream) : launch_head_bwd<kBf16, false>(a, ctas, sms, stream);
}

constexpr size_t kMaxBwdRows = 1024;  // partial rows that the workspace holds: the most CTAs of the backward

}  // namespace

int check_view(const mosaic_view* v, int B, int heads, int N, int size, View* out) {
  if (!v || !v->data || v->sb < 0 || v->sh < 0 || v->sn < 0) return MOSAIC_E_INVALID_ARG;
  constexpr long long kMost = 1ll << 37;  // a tensor copy's strides end at 2^40 bytes
  if (v->sb >= kMost || v->sh >= kMost || v->sn >= kMost) return MOSAIC_E_UNSUPPORTED;
  if (!aligned16(v->data)) return MOSAIC_E_MISALIGNED;
  out->data = (char*)v->data;
  out->sb = B > 1 ? v->sb * size : 0;
  out->sh = heads > 1 ? v->sh * size : 0;
  out->sn = N > 1 ? v->sn * size : 0;
  return (out->sb | out->sh | out->sn) & 15 ? MOSAIC_E_MISALIGNED : MOSAIC_OK;
}

namespace {
int rotary_forward(const mosaic_rotary_params* p, const mosaic_view* q, const mosaic_view* k, const float* wq, const float* wk,
                   bool norm, const int64_t* pos, int64_t pos_stride, const double* freqs, const mosaic_view* q_out,
                   const mosaic_view* k_out, void* cuda_stream) {
  int rc = check(p, norm);
  if (rc) return rc;
  if ((norm && (!wq || !wk)) || pos_stride < 0 || (p->rot_dim && (!pos || !freqs))) return MOSAIC_E_INVALID_ARG;
  HeadArgs a = base_args(p, pos, pos_stride, freqs);
  if (p->flags & MOSAIC_FLAG_INVERSE) a.amplitude = -a.amplitude;
  const int size = p->flags & MOSAIC_FLAG_FP32 ? 4 : 2;
  const mosaic_view *xs[2] = {q, k}, *ys[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) {
    HeadTensor& t = a.t[i];
    if ((rc = check_view(xs[i], p->B, t.heads, p->N, size, &t.x))) return rc;
    if ((rc = check_view(ys[i], p->B, t.heads, p->N, size, &t.y))) return rc;
    t.w = i ? wk : wq;
  }
  if (((uintptr_t)wq | (uintptr_t)wk) & 3 || ((uintptr_t)pos | (uintptr_t)freqs) & 7) return MOSAIC_E_MISALIGNED;
  if ((rc = device_ok())) return rc;
  return launch_head(a, p->flags, norm, (cudaStream_t)cuda_stream);
}
}  // namespace

}  // namespace mosaic

using namespace mosaic;

extern "C" {

int mosaic_bsa_rotary_freqs(const mosaic_rotary_scaling* s, double* freqs_host) {
  if (!s || !freqs_host || s->kind < MOSAIC_ROTARY_PLAIN || s->kind > MOSAIC_ROTARY_BANDS) return MOSAIC_E_INVALID_ARG;
  const int rot = s->rot_dim;
  if (rot < 2 || rot % 2 || !(s->theta > 1.0) || isinf(s->theta)) return MOSAIC_E_INVALID_ARG;
  if (s->kind != MOSAIC_ROTARY_PLAIN && (!(s->factor >= 1.0) || isinf(s->factor))) return MOSAIC_E_INVALID_ARG;
  if (s->kind >= MOSAIC_ROTARY_PARTS && (!(s->length > 0.0) || isinf(s->length) || !(s->slow > 0.0) || !(s->fast > s->slow) || isinf(s->fast)))
    return MOSAIC_E_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  double theta = s->theta;
  if (s->kind == MOSAIC_ROTARY_BASE && rot > 2) theta *= pow(s->factor, rot / (rot - 2.0));
  double lo = 0.0, hi = 0.0;
  if (s->kind == MOSAIC_ROTARY_PARTS) {  // the pair that turns t times in `length`: theta^(-2i/rot) length / 2 pi = t
    lo = fmax(floor(rot * log(s->length / (two_pi * s->fast)) / (2.0 * log(theta))), 0.0);
    hi = fmin(ceil(rot * log(s->length / (two_pi * s->slow)) / (2.0 * log(theta))), rot - 1.0);
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = pow(theta, -2.0 * i / rot);
    double keep = 1.0;
    if (s->kind == MOSAIC_ROTARY_LINEAR) keep = 0.0;
    if (s->kind == MOSAIC_ROTARY_PARTS) keep = 1.0 - fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
    if (s->kind == MOSAIC_ROTARY_BANDS) keep = fmin(fmax((s->length * f / two_pi - s->slow) / (s->fast - s->slow), 0.0), 1.0);
    freqs_host[i] = s->kind == MOSAIC_ROTARY_PLAIN || s->kind == MOSAIC_ROTARY_BASE ? f : f * keep + f / s->factor * (1.0 - keep);
  }
  return MOSAIC_OK;
}

int mosaic_bsa_rotary(const mosaic_rotary_params* p, const mosaic_view* q, const mosaic_view* k, const int64_t* pos,
                      int64_t pos_stride, const double* freqs, const mosaic_view* q_out, const mosaic_view* k_out,
                      void* cuda_stream) {
  return rotary_forward(p, q, k, nullptr, nullptr, false, pos, pos_stride, freqs, q_out, k_out, cuda_stream);
}

int mosaic_bsa_qk_norm(const mosaic_rotary_params* p, const mosaic_view* q, const mosaic_view* k, const float* wq,
                       const float* wk, const int64_t* pos, int64_t pos_stride, const double* freqs, const mosaic_view* q_out,
                       const mosaic_view* k_out, void* cuda_stream) {
  return rotary_forward(p, q, k, wq, wk, true, pos, pos_stride, freqs, q_out, k_out, cuda_stream);
}

size_t mosaic_bsa_qk_norm_workspace_bytes(const mosaic_rotary_params* p) {
  return check(p, true) ? 0 : kMaxBwdRows * 2 * (size_t)p->d * sizeof(float);
}

int mosaic_bsa_qk_norm_bwd(const mosaic_rotary_params* p, const mosaic_view* q, const mosaic_view* k, const float* wq,
                           const float* wk, const int64_t* pos, int64_t pos_stride, const double* freqs,
                           const mosaic_view* d_q_out, const mosaic_view* d_k_out, const mosaic_view* dq, const mosaic_view* dk,
                           float* dwq, float* dwk, void* ws, size_t ws_bytes, void* cuda_stream) {
  int rc = check(p, true);
  if (rc) return rc;
  if (!wq || !wk || !dwq || !dwk || !ws || pos_stride < 0 || (p->rot_dim && (!pos || !freqs))) return MOSAIC_E_INVALID_ARG;
  HeadArgs a = base_args(p, pos, pos_stride, freqs);
  a.amplitude = -a.amplitude;  // turns back
  const int size = p->flags & MOSAIC_FLAG_FP32 ? 4 : 2;
  const mosaic_view *xs[2] = {q, k}, *gs[2] = {d_q_out, d_k_out}, *ys[2] = {dq, dk};
  for (int i = 0; i < 2; ++i) {
    HeadTensor& t = a.t[i];
    if ((rc = check_view(xs[i], p->B, t.heads, p->N, size, &t.x))) return rc;
    if ((rc = check_view(gs[i], p->B, t.heads, p->N, size, &t.g))) return rc;
    if ((rc = check_view(ys[i], p->B, t.heads, p->N, size, &t.y))) return rc;
    t.w = i ? wk : wq;
  }
  if (((uintptr_t)wq | (uintptr_t)wk | (uintptr_t)dwq | (uintptr_t)dwk) & 3 || ((uintptr_t)pos | (uintptr_t)freqs) & 7 ||
      (uintptr_t)ws & 255)
    return MOSAIC_E_MISALIGNED;
  if (ws_bytes < mosaic_bsa_qk_norm_workspace_bytes(p)) return MOSAIC_E_WORKSPACE_TOO_SMALL;
  if ((rc = device_ok())) return rc;
  int sms = 0;
  if ((rc = launch_setup(nullptr, 0, nullptr, &sms))) return rc;
  const long long want = (a.tokens * split(a, sms) + kHeadWarps - 1) / kHeadWarps;
  const int most = kBwdCtas * sms < (int)kMaxBwdRows ? kBwdCtas * sms : (int)kMaxBwdRows;
  const int ctas = want < most ? (int)want : most;
  a.partial = (float*)ws;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  if ((rc = launch_head_bwd(a, p->flags, ctas, sms, stream))) return rc;
  return launch_kernel(weight_sum_kernel, dim3((unsigned)((2 * p->d + 31) / 32)), 1024, 0, stream, true, 0, a.partial, ctas, p->d,
                       dwq, dwk);
}

}  // extern "C"
