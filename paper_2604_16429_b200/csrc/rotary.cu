// Rotary position embedding of Q and K by token index, and the root-mean-square norm of their heads in the same pass.
//
//   forward   y = R(p f) (x * r * w),  r = 1 / sqrt(mean(x^2) + eps)  (the rotation alone: y = R(p f) x)
//   backward  g = R(-p f) dy;  dw = sum over rows of g * x * r;  dx = r * (g * w - x * r^2 * mean(g * w * x))
//
// HBM-bound: every element is read once (x and dy in the backward) and written once.  A warp has one token and walks its
// heads; a row of d channels is spread over P lanes (the power of two that holds d / 2V), each with two 16-byte pieces of V
// channels: with half pairs the two pieces hold the pairs' two sides, otherwise one lies in the first half of the head and one in the
// second, half a head apart.  So a pair never leaves its lane, a row's sums are shuffles among P lanes, and 32 / P rows go through a warp
// at a time, a few fetched ahead.
// The token's rot_dim/2 angles are the same for all its heads: the warp's lanes share them out, take the product with the
// position in half turns and its remainder in fp64 (an angle of 1e6 radians has 2^-33 of error there, 2^-4 in fp32), and leave
// (cos, sin) in shared memory, from where every lane reads the V that it needs for each row.
//
// Measured (us on the device, beside the bytes at 6543 GB/s): rotation of [2, 16 + 4 heads, 8192, 128] fp16 with 32 channels turning
// 30.6 (25.7); norm and rotation of [1, 16 + 16, 12288, 64] bf16 22.3 (15.4); its backward for [2, 16 + 4, 8192, 128] bf16 60.8 (38.5).
// The rotation is bound by HBM and a start and end of 5 us (batches of 1 KB a warp, two ahead).  The norms and their backward are at
// no limit: counters of 2 x 8192 tokens of 16 + 4 heads of 128, caches cold, show 59 and 52 % of the issue slots and 37 and 42 % of the
// DRAM's rate used, with 24 and 16 warps an SM; what is left is latency, of copies, row sums (shuffles one after the other) and stores.
// Chosen by measurement, those three in order: CTAs an SM of the forward 3 (2: 31.2, 23.7; 4: 31.2, 23.1; 6: 38.6, 35.8), batches ahead
// 2 (1: 31.2, 24.2; 3: 31.8, 24.2); CTAs an SM of the backward 2 (1: 80.2; 3: 103), batches ahead 1 (2: 61.8; 3: 64.3; held in
// registers instead of shared memory: 84).
#include <math.h>

#include "rotary.cuh"

namespace mosaic {

namespace {

constexpr int kHeadThreads = 256, kHeadWarps = kHeadThreads / 32;
constexpr int kCtas = 3, kBwdCtas = 2;  // per SM
constexpr int kDeep = 2;       // batches of rows of the backward on their way (shared memory)
constexpr size_t kBwdRing = (size_t)kHeadWarps * kDeep * 4 * 32 * 16;
constexpr int kDeepFwd = 3;    // the same of the forward, where a row comes without a gradient
constexpr size_t kFwdRing = (size_t)kHeadWarps * kDeepFwd * 2 * 32 * 16;

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
  float* partial;  // backward: [CTAs, d] sums of the weights' gradients
  long long pos_stride;
  unsigned tokens, tasks, step;  // tokens of all batch members; tasks: tokens x parts; step: warps of the grid
  int step_b, step_n;            // the step in members and tokens
  unsigned k_step;               // backward: the same for the CTAs of K's rows, which come after q_ctas of Q's
  int k_step_b, k_step_n, q_ctas;
  int N, d, rot, lanes, parts;
  float amplitude, eps, inv_d;
};

// 16 bytes of global memory to shared memory, or (bytes 0) zeros
__device__ __forceinline__ void copy_async(uint32_t dst, const char* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ float row_sum(float v, int lanes) {
  for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int V>
__device__ __forceinline__ void read_weights(const float* w, const Place& pl, float (&wa)[V], float (&wb)[V]) {
#pragma unroll
  for (int j = 0; j < V; j += 4) {  // (a lane without channels reads what it multiplies with zeros)
    const float4 x = *reinterpret_cast<const float4*>(w + (pl.on ? pl.ca : 0) + j), y = *reinterpret_cast<const float4*>(w + (pl.on ? pl.cb : 0) + j);
    wa[j] = x.x; wa[j + 1] = x.y; wa[j + 2] = x.z; wa[j + 3] = x.w;
    wb[j] = y.x; wb[j + 1] = y.y; wb[j + 2] = y.z; wb[j + 3] = y.w;
  }
}

// Where a warp is: a batch of rows of one token.  The warps of the grid take tasks (a token, or a part of its rows) in turn; with
// more than one part a token every warp has one task.
struct Spot {
  unsigned task, step;
  int step_b, step_n;
  int b, n, r0, r1;  // rows r0 .. r1 - 1 of the task are left
  bool more;
  __device__ __forceinline__ void start(const HeadArgs& a, unsigned first, int rows) {
    task = first;
    const unsigned token = task / (unsigned)a.parts, part = task - token * a.parts;
    b = (int)(token / (unsigned)a.N);
    n = (int)(token - b * (unsigned)a.N);
    more = task < a.tasks;
    r0 = (int)(rows * part / a.parts);
    r1 = (int)(rows * (part + 1) / a.parts);
  }
  __device__ __forceinline__ void stride(unsigned by, int by_b, int by_n) {
    step = by;
    step_b = by_b;
    step_n = by_n;
  }
  __device__ __forceinline__ void next(const HeadArgs& a, int rows) {
    task += step;
    more = a.parts == 1 && task < a.tasks && task >= step;
    b += step_b;
    n += step_n;
    if (n >= a.N) { n -= a.N; ++b; }
    r0 = 0;
    r1 = rows;
  }
};

// The warps walk their tasks with the next batches' rows already asked for: they land in shared memory, where every lane reads what
// it copied itself (held in registers instead, 62 us became 84 in the backward).  A token's rows are Q's heads, then K's.
template <int T, bool HALF, bool NORM, bool PART>
__global__ void __launch_bounds__(kHeadThreads, kCtas) head_kernel(const __grid_constant__ HeadArgs a) {
  constexpr int V = Vec<T>::n, SZ = Vec<T>::bytes;
  __shared__ alignas(16) Angles angles[kHeadWarps];
  __shared__ alignas(16) float weights[2][kMaxHeadDim];
  extern __shared__ uint4 ring[];  // [warp][kDeepFwd][piece][lane]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Place pl = place<T, HALF>(a, lane);
  const int heads = a.t[0].heads, rows = heads + a.t[1].heads, ca = pl.ca * SZ, ba = (pl.cb - pl.ca) * SZ;
  Spot sp, ft;  // the batch that is worked on, and the one that is asked for, kDeepFwd - 1 further
  const int zero = await_stream();
  sp.start(a, blockIdx.x * kHeadWarps + warp + zero, rows);
  sp.stride(a.step, a.step_b, a.step_n);
  ft = sp;
  const char *xq = nullptr, *xk = nullptr;  // the rows' first
  auto find = [&]() {
    xq = a.t[0].x.data + ft.b * a.t[0].x.sb + ft.n * a.t[0].x.sn + ca;
    xk = a.t[1].x.data + ft.b * a.t[1].x.sb + ft.n * a.t[1].x.sn + ca - heads * a.t[1].x.sh;
  };
  if (ft.more) find();
  const uint4* mine = ring + (warp * kDeepFwd * 2) * 32 + lane;
  const uint32_t at = (uint32_t)__cvta_generic_to_shared(mine);
  auto fetch = [&](int slot) {
    if (ft.more) {
      const int h = ft.r0 + pl.group;
      const uint32_t dst = at + slot * 2 * 32 * 16, bytes = h < ft.r1 && pl.on ? 16u : 0u;  // 0: zeros
      const char* p = !bytes ? a.t[0].x.data : h < heads ? xq + h * a.t[0].x.sh : xk + h * a.t[1].x.sh;
      copy_async(dst, p, bytes);
      copy_async(dst + 512, p + (bytes ? ba : 0), bytes);
      ft.r0 += pl.groups;
      if (ft.r0 >= ft.r1) {
        ft.next(a, rows);
        if (ft.more) find();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kDeepFwd - 1; ++i) fetch(i);
  auto position = [&](const Spot& s) { return s.more && a.rot ? __ldg(a.pos + s.b * a.pos_stride + s.n) : 0ll; };
  long long pos = position(sp);
  still_angles(a, angles[warp], lane);
  if constexpr (NORM) {
    for (int c = threadIdx.x; c < 2 * a.d; c += kHeadThreads) weights[c >= a.d][c >= a.d ? c - a.d : c] = __ldg((c < a.d ? a.t[0].w + c : a.t[1].w + (c - a.d)) + zero);
    __syncthreads();
  }
  char *yq = nullptr, *yk = nullptr;
  bool turned = false;  // the angles are this token's
  int slot = 0;
  while (sp.more) {
    fetch(slot ? slot - 1 : kDeepFwd - 1);  // where the batch before was
    if (!turned) {
      make_angles(a, a.freqs + zero, pos, angles[warp], lane);
      yq = a.t[0].y.data + sp.b * a.t[0].y.sb + sp.n * a.t[0].y.sn + ca;
      yk = a.t[1].y.data + sp.b * a.t[1].y.sb + sp.n * a.t[1].y.sn + ca - heads * a.t[1].y.sh;
      turned = true;
      Spot after = sp;
      after.next(a, rows);
      pos = position(after);  // (asked for a token ahead)
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kDeepFwd - 1) : "memory");
    uint4 va = mine[(slot * 2 + 0) * 32], vb = mine[(slot * 2 + 1) * 32];
    float fa[V], fb[V];
    widen<T>(va, fa);
    widen<T>(vb, fb);
    slot = slot + 1 == kDeepFwd ? 0 : slot + 1;
    const int h = sp.r0 + pl.group;
    const bool there = h < sp.r1;
    sp.r0 += pl.groups;
    if (sp.r0 >= sp.r1) {
      sp.next(a, rows);
      turned = false;
    }
    if constexpr (NORM) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) ss = fmaf(fa[j], fa[j], fmaf(fb[j], fb[j], ss));
      const float rr = rsqrtf(row_sum(ss, a.lanes) * a.inv_d + a.eps);
      float ga[V], gb[V];
      read_weights<V>(weights[h >= heads], pl, ga, gb);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        fa[j] *= rr * ga[j];
        fb[j] *= rr * gb[j];
      }
    }
    if constexpr (PART && !NORM) {
      turn_part<T, HALF>(va, vb, angles[warp], a, pl);
    } else {
      turn<V, HALF, PART>(fa, fb, angles[warp], a, pl);
    }
    if (there && pl.on) {
      char* y = h < heads ? yq + h * a.t[0].y.sh : yk + h * a.t[1].y.sh;
      *reinterpret_cast<uint4*>(y) = PART && !NORM ? va : narrow<T>(fa);
      *reinterpret_cast<uint4*>(y + ba) = PART && !NORM ? vb : narrow<T>(fb);
    }
  }
}

// The sums of the weights' gradients stay in registers over a CTA's tokens (a lane has the same channels in every row); the first
// CTAs have Q's rows, the others K's, and each leaves one row of partial sums.  Packed fp32 arithmetic: the pass is as much bound
// by instructions as by memory.
template <int T, bool HALF, bool PART>
__global__ void __launch_bounds__(kHeadThreads, kBwdCtas) head_bwd_kernel(const __grid_constant__ HeadArgs a) {
  constexpr int V = Vec<T>::n, SZ = Vec<T>::bytes, P = V / 2;
  __shared__ alignas(16) Angles angles[kHeadWarps];
  __shared__ alignas(16) float weights[kMaxHeadDim];
  __shared__ float sums[kHeadWarps][kMaxHeadDim];
  extern __shared__ uint4 ring[];  // [warp][kDeep][x, x, g, g][lane]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Place pl = place<T, HALF>(a, lane);
  const bool keys = (int)blockIdx.x >= a.q_ctas;
  const HeadTensor& t = a.t[keys];
  const int ca = pl.ca * SZ, ba = (pl.cb - pl.ca) * SZ, cta = (int)blockIdx.x - (keys ? a.q_ctas : 0);
  Spot sp, ft;  // the batch that is worked on, and the one that is asked for, kDeep - 1 further
  const int zero = await_stream();
  sp.start(a, cta * kHeadWarps + warp + zero, t.heads);
  if (keys) sp.stride(a.k_step, a.k_step_b, a.k_step_n);
  else sp.stride(a.step, a.step_b, a.step_n);
  ft = sp;
  const char *x = nullptr, *g = nullptr;  // this lane's next row
  char* y = nullptr;
  const long long ox = pl.group * t.x.sh + ca, og = pl.group * t.g.sh + ca, oy = pl.group * t.y.sh + ca;
  const long long jx = pl.groups * t.x.sh, jg = pl.groups * t.g.sh, jy = pl.groups * t.y.sh;
  auto find = [&]() {
    x = t.x.data + ft.b * t.x.sb + ft.n * t.x.sn + ft.r0 * t.x.sh + ox;
    g = t.g.data + ft.b * t.g.sb + ft.n * t.g.sn + ft.r0 * t.g.sh + og;
  };
  if (ft.more) find();
  const uint4* mine = ring + (warp * kDeep * 4) * 32 + lane;  // (a lane reads what it copied itself)
  const uint32_t at = (uint32_t)__cvta_generic_to_shared(mine);
  auto fetch = [&](int slot) {
    if (ft.more) {
      const uint32_t dst = at + slot * 4 * 32 * 16, bytes = ft.r0 + pl.group < ft.r1 && pl.on ? 16u : 0u;  // 0: zeros
      const char *p = bytes ? x : t.x.data, *q = bytes ? g : t.g.data;
      copy_async(dst, p, bytes);
      copy_async(dst + 512, p + (bytes ? ba : 0), bytes);
      copy_async(dst + 1024, q, bytes);
      copy_async(dst + 1536, q + (bytes ? ba : 0), bytes);
      ft.r0 += pl.groups;
      if (ft.r0 >= ft.r1) {
        ft.next(a, t.heads);
        if (ft.more) find();
      } else {
        x += jx;
        g += jg;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kDeep - 1; ++i) fetch(i);
  auto position = [&](const Spot& s) { return s.more && a.rot ? __ldg(a.pos + s.b * a.pos_stride + s.n) : 0ll; };
  long long pos = position(sp);
  still_angles(a, angles[warp], lane);
  for (int c = threadIdx.x; c < a.d; c += kHeadThreads) weights[c] = __ldg(t.w + c + zero);
  __syncthreads();
  uint64_t da[P], db[P];
#pragma unroll
  for (int j = 0; j < P; ++j) da[j] = db[j] = 0ull;
  bool turned = false;
  int slot = 0;
  while (sp.more) {
    fetch(slot ? slot - 1 : kDeep - 1);  // where the batch before was
    asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 1) : "memory");
    float ha[V], hb[V], fa[V], fb[V];
    widen<T>(mine[(slot * 4 + 0) * 32], fa);
    widen<T>(mine[(slot * 4 + 1) * 32], fb);
    widen<T>(mine[(slot * 4 + 2) * 32], ha);
    widen<T>(mine[(slot * 4 + 3) * 32], hb);
    slot = slot + 1 == kDeep ? 0 : slot + 1;
    const bool there = sp.r0 + pl.group < sp.r1;
    if (!turned) {
      make_angles(a, a.freqs + zero, pos, angles[warp], lane);
      y = t.y.data + sp.b * t.y.sb + sp.n * t.y.sn + sp.r0 * t.y.sh + oy;
      turned = true;
      Spot after = sp;
      after.next(a, t.heads);
      pos = position(after);  // (asked for a token ahead)
    }
    char* out = y;
    y += jy;
    sp.r0 += pl.groups;
    if (sp.r0 >= sp.r1) {
      sp.next(a, t.heads);
      turned = false;
    }
    turn<V, HALF, PART>(ha, hb, angles[warp], a, pl);
    float wa[V], wb[V];
    read_weights<V>(weights, pl, wa, wb);
    uint64_t ss2 = 0ull, dot2 = 0ull, wh[V];  // wh: the weighted gradient
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint64_t f0 = pack2(fa[2 * j], fa[2 * j + 1]), f1 = pack2(fb[2 * j], fb[2 * j + 1]);
      wh[j] = mul2(pack2(ha[2 * j], ha[2 * j + 1]), pack2(wa[2 * j], wa[2 * j + 1]));
      wh[P + j] = mul2(pack2(hb[2 * j], hb[2 * j + 1]), pack2(wb[2 * j], wb[2 * j + 1]));
      ss2 = fma2(f0, f0, fma2(f1, f1, ss2));
      dot2 = fma2(wh[j], f0, fma2(wh[P + j], f1, dot2));
    }
    float s0, s1, d0, d1;
    unpack2(ss2, s0, s1);
    unpack2(dot2, d0, d1);
    const float ss = row_sum(s0 + s1, a.lanes), dot = row_sum(d0 + d1, a.lanes);
    const float rr = there ? rsqrtf(ss * a.inv_d + a.eps) : 0.f;  // (of zeros that are no row it may be infinite)
    const uint64_t rr2 = pack2(rr, rr), back2 = pack2(-dot * rr * rr * a.inv_d, -dot * rr * rr * a.inv_d);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint64_t t0 = mul2(pack2(fa[2 * j], fa[2 * j + 1]), rr2), t1 = mul2(pack2(fb[2 * j], fb[2 * j + 1]), rr2);
      da[j] = fma2(pack2(ha[2 * j], ha[2 * j + 1]), t0, da[j]);
      db[j] = fma2(pack2(hb[2 * j], hb[2 * j + 1]), t1, db[j]);
      unpack2(fma2(t0, back2, mul2(wh[j], rr2)), fa[2 * j], fa[2 * j + 1]);
      unpack2(fma2(t1, back2, mul2(wh[P + j], rr2)), fb[2 * j], fb[2 * j + 1]);
    }
    if (there && pl.on) {
      *reinterpret_cast<uint4*>(out) = narrow<T>(fa);
      *reinterpret_cast<uint4*>(out + ba) = narrow<T>(fb);
    }
  }
  // lane groups, then warps, each in a fixed order
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float u, v, lo, hi;
    unpack2(da[j / 2], lo, hi);
    u = j & 1 ? hi : lo;
    unpack2(db[j / 2], lo, hi);
    v = j & 1 ? hi : lo;
    for (int o = a.lanes; o < 32; o <<= 1) {
      u += __shfl_xor_sync(0xffffffffu, u, o);
      v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    if (pl.group == 0 && pl.on) {
      sums[warp][pl.ca + j] = u;
      sums[warp][pl.cb + j] = v;
    }
  }
  __syncthreads();
  if ((int)threadIdx.x < a.d) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kHeadWarps; ++w) v += sums[w][threadIdx.x];
    a.partial[(long long)blockIdx.x * a.d + threadIdx.x] = v;
  }
}

// Sums of the CTAs' partial rows, Q's and K's: 32 columns a CTA, 32 threads a column, joined in a fixed order.
__global__ void __launch_bounds__(1024) weight_sum_kernel(const float* __restrict__ partial, int q_rows, int k_rows, int d,
                                                          float* __restrict__ dwq, float* __restrict__ dwk) {
  __shared__ float part[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c0 = blockIdx.x * 32, col = c0 + x;
  const bool keys = blockIdx.y != 0;
  partial += await_stream() + (keys ? (long long)q_rows * d : 0);
  float v = 0.f;
  if (col < d)
    for (int r = y; r < (keys ? k_rows : q_rows); r += 32) v += partial[(long long)r * d + col];
  part[y][x] = v;
  __syncthreads();
  v = part[x][y];  // a warp per column now
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (x == 0 && c0 + y < d) (keys ? dwk : dwq)[c0 + y] = v;
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
  if ((long long)p->B * p->N > (1 << 30) || (long long)p->H + p->Hkv > (1 << 16)) return MOSAIC_E_UNSUPPORTED;
  return MOSAIC_OK;
}

HeadArgs base_args(const mosaic_rotary_params* p, const int64_t* pos, int64_t pos_stride, const double* freqs) {
  HeadArgs a = {};
  a.pos = pos;
  a.freqs = freqs;
  a.pos_stride = pos_stride;
  a.tokens = (unsigned)((long long)p->B * p->N);
  a.N = p->N;
  a.d = p->d;
  a.rot = p->rot_dim;
  const int v = p->flags & MOSAIC_FLAG_FP32 ? 4 : 8;
  for (a.lanes = 1; a.lanes * 2 * v < p->d;) a.lanes *= 2;
  a.amplitude = p->amplitude > 0.f ? p->amplitude : 1.f;
  a.eps = p->eps;
  a.inv_d = 1.f / (float)p->d;
  a.t[0].heads = p->H;
  a.t[1].heads = p->Hkv;
  return a;
}

// The grid: as many CTAs as there are tasks, or, one task a token, `ctas` at the most.
int spread(HeadArgs* a, long long ctas) {
  a->tasks = a->tokens * a->parts;
  long long blocks = ((long long)a->tasks + kHeadWarps - 1) / kHeadWarps;
  if (a->parts == 1 && blocks > ctas) blocks = ctas;
  a->step = (unsigned)blocks * kHeadWarps;
  a->step_b = (int)(a->step / (unsigned)a->N);
  a->step_n = (int)(a->step % (unsigned)a->N);
  return (int)blocks;
}

// Few tokens: a token's `rows` rows go to several warps, until there are sixteen warps an SM or a warp has one round of rows.
int plan(HeadArgs* a, int rows, int sms, long long ctas) {
  a->parts = 1;
  while ((long long)a->tokens * a->parts < 16ll * sms && a->parts * (32 / a->lanes) < rows) a->parts *= 2;
  return spread(a, ctas);
}

template <int T, bool HALF, bool NORM, bool PART>
int launch_head(HeadArgs a, cudaStream_t stream) {
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup(reinterpret_cast<const void*>(head_kernel<T, HALF, NORM, PART>), kFwdRing, &configured, &sms)) return rc;
  const int blocks = plan(&a, a.t[0].heads + a.t[1].heads, sms, (long long)kCtas * sms);
  return launch_kernel(head_kernel<T, HALF, NORM, PART>, dim3((unsigned)blocks), kHeadThreads, kFwdRing, stream, true, 0, a);
}
template <int T, bool HALF>
int launch_head(const HeadArgs& a, bool norm, cudaStream_t stream) {
  const bool part = a.rot < a.d;
  if (norm) return part ? launch_head<T, HALF, true, true>(a, stream) : launch_head<T, HALF, true, false>(a, stream);
  return part ? launch_head<T, HALF, false, true>(a, stream) : launch_head<T, HALF, false, false>(a, stream);
}
int launch_head(const HeadArgs& a, uint32_t flags, bool norm, cudaStream_t stream) {
  const bool half = (flags & MOSAIC_FLAG_HALF_PAIRS) != 0;
  if (flags & MOSAIC_FLAG_FP32) return half ? launch_head<kF32, true>(a, norm, stream) : launch_head<kF32, false>(a, norm, stream);
  if (flags & MOSAIC_FLAG_FP16) return half ? launch_head<kF16, true>(a, norm, stream) : launch_head<kF16, false>(a, norm, stream);
  return half ? launch_head<kBf16, true>(a, norm, stream) : launch_head<kBf16, false>(a, norm, stream);
}

template <int T, bool HALF, bool PART>
int launch_head_bwd(const HeadArgs& a, int ctas, cudaStream_t stream) {
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup(reinterpret_cast<const void*>(head_bwd_kernel<T, HALF, PART>), kBwdRing, &configured, &sms)) return rc;
  return launch_kernel(head_bwd_kernel<T, HALF, PART>, dim3((unsigned)ctas), kHeadThreads, kBwdRing, stream, true, 0, a);
}
template <int T>
int launch_head_bwd(const HeadArgs& a, bool half, int ctas, cudaStream_t stream) {
  const bool part = a.rot < a.d;
  if (half) return part ? launch_head_bwd<T, true, true>(a, ctas, stream) : launch_head_bwd<T, true, false>(a, ctas, stream);
  return part ? launch_head_bwd<T, false, true>(a, ctas, stream) : launch_head_bwd<T, false, false>(a, ctas, stream);
}
int launch_head_bwd(const HeadArgs& a, uint32_t flags, int ctas, cudaStream_t stream) {
  const bool half = (flags & MOSAIC_FLAG_HALF_PAIRS) != 0;
  if (flags & MOSAIC_FLAG_FP32) return launch_head_bwd<kF32>(a, half, ctas, stream);
  return flags & MOSAIC_FLAG_FP16 ? launch_head_bwd<kF16>(a, half, ctas, stream) : launch_head_bwd<kBf16>(a, half, ctas, stream);
}

constexpr size_t kMaxBwdRows = 2048;  // partial rows that the workspace holds: the most CTAs of the backward

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
  return check(p, true) ? 0 : kMaxBwdRows * (size_t)p->d * sizeof(float);
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
  // CTAs in the ratio of the work: a token's rows by rounds of the warp, and its angles as much as two rounds
  const int groups = 32 / a.lanes, work_q = 2 + (p->H + groups - 1) / groups, work_k = 2 + (p->Hkv + groups - 1) / groups, most = kBwdCtas * sms;
  const int most_q = most * work_q / (work_q + work_k) > 0 ? most * work_q / (work_q + work_k) : 1;
  HeadArgs k_plan = a;
  a.q_ctas = plan(&a, p->H, sms, most_q);
  k_plan.parts = a.parts;
  const int k_ctas = spread(&k_plan, most - most_q > 0 ? most - most_q : 1), ctas = a.q_ctas + k_ctas;
  a.k_step = k_plan.step;
  a.k_step_b = k_plan.step_b;
  a.k_step_n = k_plan.step_n;
  if (ctas > (int)kMaxBwdRows) return MOSAIC_E_UNSUPPORTED;
  a.partial = (float*)ws;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  if ((rc = launch_head_bwd(a, p->flags, ctas, stream))) return rc;
  return launch_kernel(weight_sum_kernel, dim3((unsigned)((p->d + 31) / 32), 2u), 1024, 0, stream, true, 0, a.partial, a.q_ctas, k_ctas,
                       p->d, dwq, dwk);
}

}  // extern "C"
