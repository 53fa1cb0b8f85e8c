// Attention of one or a few new tokens per sequence over a paged cache, and the join of its parts.
//
//   o_i = sum_j exp(scale q_i . k_j - m_i) v_j / l_i  over the keys that row i sees: j <= p_i, and p_i - j < window or j < sinks
// HBM-bound: the visible keys and values of a key/value head are read once for all rows (new tokens x query heads of the group, up to
// 16 at a time).  The keys of a member are cut into chunks of 512; a chunk of a head is an item.  Persistent CTAs, one an SM, take
// equal shares of the list of all items, which each works out from the lengths; a CTA's items lie one after the other, so that a member's
// queries stay in registers.
//
// A warp takes every eighth step of 16 keys of the chunk.  It asks for its own steps by TMA (pages are multiples of 16 slots, so a step
// lies in one; the page numbers of an item's steps are looked up an item ahead) into a ring of its own, and goes on asking into
// the next items, so that the memory never waits for a chunk's end.  Products of 16 x 8 x 16 are enough:
//   S^T = K Q^T (16 keys x 8 rows), O^T += V^T P^T (16 channels x 8 rows), P^T turned from accumulator to operand by a transpose
// Weights round to 16 bits once, as operands; everything else is fp32.  The warps' maxima, sums and accumulators are joined through
// shared memory at the chunk's end, and leave as a part; a second kernel joins a row's parts in their order.
#include <type_traits>

#include "mma16.cuh"
#include "paged.cuh"

namespace mosaic {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kStep = 16, kWarpSteps = kChunkKeys / (kStep * kWarps);

// NT: tiles of 8 rows that a CTA takes
template <int D, int NT>
struct Smem {
  static constexpr int kHalf = kStep * D * 2, kStepBytes = 2 * kHalf;  // a step's keys, then its values
  static constexpr int kStages = (NT == 1 ? 196608 : 131072) / (kWarps * kStepBytes);
  static constexpr int kPitch = D + 4;  // of a row of part_o: lanes that store side by side meet different banks
  unsigned char ring[kWarps][kStages][kStepBytes];
  float part_o[kWarps][8 * NT][kPitch], part_m[kWarps][8 * NT], part_l[kWarps][8 * NT];
  unsigned long long full[kWarps][kStages];
  int hole[kWarps][kStages];  // the step's page is not there
  int scan[kWarps + 1], start[2];
  int abort;
};

struct DecArgs {
  View q, o;
  float* lse;
  PartsOut parts;
  int blocks;  // of rows
  bool direct, clear;
  int* status;
};

// A place in the list of all items: members, their heads, their parts, blocks of rows
struct Walk {
  Parts p;
  int b, hk, o, rb;
  __device__ __forceinline__ void member(const PagedGeo& g, const DecArgs& a) {
    p = parts_of(g, b);
    if (a.direct) p.n = p.ql > 0 ? 1 : 0;  // (a member without keys has results too)
  }
  __device__ __forceinline__ void next(const PagedGeo& g, const DecArgs& a) {
    if (++rb < a.blocks) return;
    rb = 0;
    if (++o < p.n) return;
    o = 0;
    if (++hk < g.Hkv) return;
    hk = 0;
    do {
      if (++b >= g.B) return;
      member(g, a);
    } while (p.n == 0);
  }
  __device__ __forceinline__ int step(int warp, int i) const { return chunk_of(p, o) * kChunkKeys + (warp + kWarps * i) * kStep; }
  // any row sees some of the step's keys
  __device__ __forceinline__ bool seen(int j0) const { return j0 < p.kl && (j0 + kStep > p.from || j0 < p.sinks); }
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// Sum of v over the threads before this one, and over all
__device__ __forceinline__ int block_scan(int v, int* scan, int& total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) scan[warp] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    before += w < warp ? scan[w] : 0;
    total += scan[w];
  }
  __syncthreads();
  return before + x - v;
}

template <int D, bool F16, int NT>
__global__ void __launch_bounds__(kThreads, 1)
    paged_parts_kernel(const PagedGeo g, const __grid_constant__ DecArgs a, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v) {
  using S = Smem<D, NT>;
  constexpr int kRowsCta = 8 * NT, kStages = S::kStages;
  extern __shared__ unsigned char smem_raw[];
  S& sm = *reinterpret_cast<S*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gq = lane >> 2, tq = lane & 3;
  if (tid == 0) {
    for (int w = 0; w < kWarps; ++w)
      for (int s = 0; s < kStages; ++s) mbar_init(s32(&sm.full[w][s]), 1);
    sm.abort = 0;
    cta_publish_barriers();
  }
  __syncthreads();
  const int zero = await_stream();
  // A code is written no earlier than a wait's bound of seconds after its CTA began; the first CTA has cleared the word by then.
  if (a.clear && blockIdx.x == 0 && tid == 0) a.status[zero] = 0;

  // ---- this CTA's share of the list
  const int per = g.Hkv * a.blocks;
  Walk w;
  int left, total = 0, before = 0;
  {
    auto items = [&](int b) {
      w.b = b;
      if (b >= g.B) return 0;
      w.member(g, a);
      return w.p.n * per;
    };
    for (int b0 = 0; b0 < g.B; b0 += kThreads) {
      int all;
      before = block_scan(items(b0 + tid + zero), sm.scan, all);
      total += all;
    }
    const int lo = (int)((long long)total * blockIdx.x / gridDim.x), hi = (int)((long long)total * (blockIdx.x + 1) / gridDim.x);
    left = hi - lo;
    if (left == 0) return;
    int base = 0;
    for (int b0 = 0; b0 < g.B; b0 += kThreads) {
      int all = 0;
      if (g.B > kThreads) before = block_scan(items(b0 + tid + zero), sm.scan, all);
      const int n = w.b < g.B ? w.p.n * per : 0, at = lo - base - before;
      if (at >= 0 && at < n) {
        sm.start[0] = w.b;
        sm.start[1] = at;
      }
      base += all;
    }
    __syncthreads();
    w.b = sm.start[0];
    w.member(g, a);
    const int at = sm.start[1], r = at % (w.p.n * a.blocks);
    w.hk = at / (w.p.n * a.blocks);
    w.o = r / a.blocks;
    w.rb = r % a.blocks;
  }

  // ---- the warp's steps on their way: an item is looked up while the one before is asked for
  Walk look = w;
  int looked = left, f_hk = 0, f_at = 0, f_id = 0, n_hk = 0, n_at = 0, n_id = 0, slot_in = 0;
  unsigned f_mask = 0, n_mask = 0;
  bool more = true, ok = true;
  uint32_t issued = 0, taken = 0;
  auto look_up = [&]() {
    more = looked > 0;
    if (!more) return;
    const int j0 = look.step(warp, lane & (kWarpSteps - 1));
    const bool seen = lane < kWarpSteps && look.seen(j0);
    n_mask = __ballot_sync(0xffffffffu, seen);
    n_id = seen ? __ldg(g.table + look.b * g.table_stride + (j0 >> g.shift)) : -1;
    n_hk = look.hk;
    n_at = look.step(warp, 0);
    --looked;
    if (looked > 0) look.next(g, a);
  };
  look_up();
  auto fetch = [&]() {
#ifdef MOSAIC_TEST_WITHHOLD_FIRST_LIST
    return;  // test build only: nothing is ever loaded, so that every wait for it runs out
#endif
    while (f_mask == 0) {
      if (!more) return;
      f_mask = n_mask;
      f_hk = n_hk;
      f_at = n_at;
      f_id = n_id;
      look_up();
    }
    const int i = __ffs(f_mask) - 1;
    f_mask &= f_mask - 1;
    const int id = __shfl_sync(0xffffffffu, f_id, i);
    if (lane == 0) {
      const bool hole = (unsigned)id >= (unsigned)g.pages;
      const int page = hole ? g.pages : id;  // (rows behind the last page arrive as zeros)
      const int slot = (f_at + kWarps * kStep * i) & ((1 << g.shift) - 1);
      const uint32_t bar = s32(&sm.full[warp][slot_in]), dst = s32(sm.ring[warp][slot_in]);
      sm.hole[warp][slot_in] = hole;
      mbar_expect_tx(bar, S::kStepBytes);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) tma_load_4d(dst + c * kStep * 128, &map_k, bar, 64 * c, slot, f_hk, page);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) tma_load_4d(dst + S::kHalf + c * kStep * 128, &map_v, bar, 64 * c, slot, f_hk, page);
    }
    __syncwarp();
    slot_in = slot_in + 1 == kStages ? 0 : slot_in + 1;
    ++issued;
  };
#pragma unroll 1
  for (int s = 0; s < kStages; ++s) fetch();

  // ---- items
  int slot_out = 0, phase = 0, have_b = -1, have_hk = -1, have_rb = -1;
  uint32_t qf[NT][D / 16][2];
  const int rows = g.G * g.T;
  const uint32_t ka = (uint32_t)((lane & 15) * 128), kx = (uint32_t)(lane & 7), kh = (uint32_t)(lane >> 4);           // keys as they lie
  const uint32_t va = (uint32_t)(((lane & 7) + 8 * (lane >> 4)) * 128), vh = (uint32_t)((lane >> 3) & 1);             // values transposed
#pragma unroll 1
  for (; left > 0; --left) {
    if (w.b != have_b || w.hk != have_hk || w.rb != have_rb) {
      have_b = w.b; have_hk = w.hk; have_rb = w.rb;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = w.rb * kRowsCta + 8 * nt + gq, i = r / g.G, h = r - i * g.G;
        const char* src = a.q.data + w.b * a.q.sb + (w.hk * g.G + h) * a.q.sh + i * a.q.sn + 4 * tq;
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
          for (int x = 0; x < 2; ++x) qf[nt][c][x] = r < rows ? __ldg(reinterpret_cast<const unsigned*>(src + 32 * c + 16 * x)) : 0u;
      }
    }
    // the last key that the lane's rows see (8 nt + 2 tq + x), -1 where there is no such row
    int last[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = w.rb * kRowsCta + 8 * nt + 2 * tq + x, i = r / g.G;
        last[nt][x] = r < rows && i < w.p.ql ? w.p.p0 + i : -1;
      }
    float m[NT][2], l[NT][2], acc[NT][D / 16][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) acc[nt][c][0] = acc[nt][c][1] = acc[nt][c][2] = acc[nt][c][3] = 0.f;
    }
#pragma unroll 1
    for (int i = 0; i < kWarpSteps; ++i) {
      const int j0 = w.step(warp, i);
      if (!ok || !w.seen(j0)) continue;
      ok = warp_wait(s32(&sm.full[warp][slot_out]), phase, &sm.abort, a.status);
      if (!ok) continue;
      const uint32_t kt = s32(sm.ring[warp][slot_out]), vt = kt + S::kHalf;
      if (!sm.hole[warp][slot_out]) {
        // all rows see all of the step
        const bool whole = j0 + kStep - 1 <= w.p.p0 && (!g.window || j0 >= w.p.kl - g.window || j0 + kStep <= w.p.sinks);
        if (!whole) {  // a weight of zero does not silence what is no number: values that no row sees become zeros
          for (int r = 0; r < kStep; ++r) {
            const int j = j0 + r;
            if ((j >= w.p.kl || (j < w.p.from && j >= w.p.sinks)) && lane < D / 8)
              *reinterpret_cast<uint4*>(sm.ring[warp][slot_out] + S::kHalf + (lane >> 3) * kStep * 128 + r * 128 + (lane & 7) * 16) =
                  make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (the next copy into the slot comes after these stores)
          __syncwarp();
        }
        float s[NT][2][4];  // in two chains
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) s[nt][x][0] = s[nt][x][1] = s[nt][x][2] = s[nt][x][3] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          uint32_t f[4];
          ldsm4(f, kt + (c >> 2) * kStep * 128 + ka + (((2 * (c & 3) + kh) ^ kx) << 4));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16816<F16>(s[nt][c & 1], f[0], f[1], f[2], f[3], qf[nt][c][0], qf[nt][c][1]);
        }
        uint32_t pt[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float z[4];  // (key gq, row 2 tq), (gq, 2 tq + 1), (gq + 8, 2 tq), (gq + 8, 2 tq + 1)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            z[x] = (s[nt][0][x] + s[nt][1][x]) * g.scale_log2;
            if (!whole) {
              const int j = j0 + gq + 4 * (x & 2), p = last[nt][x & 1];
              if (j > p || (g.window && p - j >= g.window && j >= w.p.sinks)) z[x] = -INFINITY;
            }
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float mx = fmaxf(z[x], z[x + 2]);
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            if (mx > m[nt][x]) {  // (the same in the eight lanes of the row)
              const float alpha = ex2(m[nt][x] - mx);
              m[nt][x] = mx;
              l[nt][x] *= alpha;
#pragma unroll
              for (int c = 0; c < D / 16; ++c) {
                acc[nt][c][x] *= alpha;
                acc[nt][c][x + 2] *= alpha;
              }
            }
            const float ref = m[nt][x] == -INFINITY ? 0.f : m[nt][x];  // (nothing seen so far)
            z[x] = ex2(z[x] - ref);
            z[x + 2] = ex2(z[x + 2] - ref);
            l[nt][x] += z[x] + z[x + 2];
          }
          pt[nt][0] = transpose8(pack2<F16>(z[0], z[1]));
          pt[nt][1] = transpose8(pack2<F16>(z[2], z[3]));
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          uint32_t f[4];
          ldsm4t(f, vt + (c >> 2) * kStep * 128 + va + (((2 * (c & 3) + vh) ^ kx) << 4));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16816<F16>(acc[nt][c], f[0], f[1], f[2], f[3], pt[nt][0], pt[nt][1]);
        }
      }
      __syncwarp();  // the slot has been read
      ++taken;
      if (++slot_out == kStages) { slot_out = 0; phase ^= 1; }
      fetch();
    }

    // the warps' parts
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float sum = l[nt][x];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        const int h = 8 * nt + 2 * tq + x;
        if (gq == 0) {
          sm.part_m[warp][h] = m[nt][x];
          sm.part_l[warp][h] = sum;
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          sm.part_o[warp][h][16 * c + gq] = acc[nt][c][x];
          sm.part_o[warp][h][16 * c + gq + 8] = acc[nt][c][x + 2];
        }
      }
    __syncthreads();
    for (int e = tid; e < kRowsCta * D / 4; e += kThreads) {
      const int h = e / (D / 4), c = 4 * (e - h * (D / 4)), r = w.rb * kRowsCta + h, i = r / g.G;
      if (r >= rows || i >= w.p.ql) continue;
      float mx = -INFINITY, sum = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int y = 0; y < kWarps; ++y) mx = fmaxf(mx, sm.part_m[y][h]);
#pragma unroll
      for (int y = 0; y < kWarps; ++y) {
        const float f = sm.part_m[y][h] == -INFINITY ? 0.f : ex2(sm.part_m[y][h] - mx);
        const float4 u = *reinterpret_cast<const float4*>(&sm.part_o[y][h][c]);
        sum = fmaf(sm.part_l[y][h], f, sum);
        v.x = fmaf(u.x, f, v.x);
        v.y = fmaf(u.y, f, v.y);
        v.z = fmaf(u.z, f, v.z);
        v.w = fmaf(u.w, f, v.w);
      }
      const int head = w.hk * g.G + r - i * g.G;
      const long long row = ((long long)w.b * g.H + head) * g.T + i;
      if (a.direct) {
        const bool some = !(sum <= 0.f);  // (a sum that is not a number stays one)
        const float inv = some ? 1.f / sum : 0.f;
        *reinterpret_cast<uint2*>(a.o.data + w.b * a.o.sb + head * a.o.sh + i * a.o.sn + 2 * c) =
            make_uint2(pack2<F16>(v.x * inv, v.y * inv), pack2<F16>(v.z * inv, v.w * inv));
        if (c == 0) a.lse[row] = some ? (mx + log2f(sum)) * 0.6931471805599453f : -INFINITY;
      } else {
        const long long at = (long long)(a.parts.shared + w.o) * a.parts.rows + row;
        *reinterpret_cast<float4*>(a.parts.o + at * D + c) = v;
        if (c == 0) a.parts.ml[at] = make_float2(mx, sum);
      }
    }
    __syncthreads();  // the parts have been read
    w.next(g, a);
  }
  // copies must have landed before the CTA's memory is released
  if (!ok && lane == 0)
    for (; taken < issued; ++taken) {
      mbar_drain(s32(&sm.full[warp][slot_out]), phase);
      if (++slot_out == kStages) { slot_out = 0; phase ^= 1; }
    }
}

// A row's parts in their order: W warps share them out, part p to warp p % W, and are joined in turn.
template <int D, bool F16, int W>
__global__ void __launch_bounds__(kThreads) paged_join_kernel(const PagedGeo g, const PartsOut in, const View o, float* __restrict__ lse) {
  constexpr int V = D / 32;  // channels of a lane
  __shared__ float part_o[kWarps][D], part_l[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp % W;
  const long long row = (long long)blockIdx.x * (kWarps / W) + warp / W + await_stream();
  bool live = row < in.rows;
  const int i = (int)(row % g.T), head = (int)(row / g.T % g.H), b = live ? (int)(row / g.T / g.H) : 0;
  const Parts p = parts_of(g, b);
  live = live && i < p.ql;
  const int n = live ? in.shared + p.n : 0;
  float mx = -INFINITY, sum = 0.f, v[V];
#pragma unroll
  for (int x = 0; x < V; ++x) v[x] = 0.f;
  for (int y = lane; y < n; y += 32) mx = fmaxf(mx, __ldcg(&in.ml[y * in.rows + row].x));
#pragma unroll
  for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
#pragma unroll 4
  for (int y = w; y < n; y += W) {
    const long long at = y * in.rows + row;
    const float2 ml = __ldcg(in.ml + at);
    const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - mx);
    const float* src = in.o + at * D + V * lane;
    float u[V];
    if constexpr (V == 4) {
      const float4 t = __ldcg(reinterpret_cast<const float4*>(src));
      u[0] = t.x; u[1] = t.y; u[2] = t.z; u[3] = t.w;
    } else {
      const float2 t = __ldcg(reinterpret_cast<const float2*>(src));
      u[0] = t.x; u[1] = t.y;
    }
    sum = fmaf(ml.y, f, sum);
#pragma unroll
    for (int x = 0; x < V; ++x) v[x] = fmaf(u[x], f, v[x]);
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int x = 0; x < V; ++x) part_o[warp][V * lane + x] = v[x];
    if (lane == 0) part_l[warp] = sum;
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int y = 1; y < W; ++y) {
      sum += part_l[warp + y];
#pragma unroll
      for (int x = 0; x < V; ++x) v[x] += part_o[warp + y][V * lane + x];
    }
  }
  if (!live) return;
  const bool some = !(sum <= 0.f);
  const float inv = some ? 1.f / sum : 0.f;
  char* dst = o.data + b * o.sb + head * o.sh + i * o.sn + 2 * V * lane;
  if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<F16>(v[0] * inv, v[1] * inv), pack2<F16>(v[2] * inv, v[3] * inv));
  else *reinterpret_cast<uint32_t*>(dst) = pack2<F16>(v[0] * inv, v[1] * inv);
  if (lane == 0) lse[row] = some ? (mx + log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool F16, int NT>
int launch_parts(const HostCtx& c, const PagedGeo& g, DecArgs a, const View& k_pages, const View& v_pages, int most_parts) {
  CUtensorMap mk, mv;
  if (!make_map_pool(&mk, k_pages, g, kStep) || !make_map_pool(&mv, v_pages, g, kStep)) return MOSAIC_E_CUDA;
  const size_t smem = sizeof(Smem<D, NT>) + 1024;
  static_assert(sizeof(Smem<D, NT>) + 1024 <= 232448, "more shared memory than a CTA can have");
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup(reinterpret_cast<const void*>(paged_parts_kernel<D, F16, NT>), smem, &configured, &sms)) return rc;
  a.blocks = (g.G * g.T + 8 * NT - 1) / (8 * NT);
  const long long most = (long long)g.B * g.Hkv * a.blocks * most_parts;
  if (most > 0x7fffffffll) return MOSAIC_E_UNSUPPORTED;
  return launch_kernel(paged_parts_kernel<D, F16, NT>, dim3((unsigned)(most < sms ? most : sms)), kThreads, smem, c.stream, true, 0, g, a, mk, mv);
}

template <int D, bool F16, int W>
int launch_join(const HostCtx& c, const PagedGeo& g, const PartsOut& parts, const View& o, float* lse) {
  constexpr int per = kWarps / W;
  return launch_kernel(paged_join_kernel<D, F16, W>, dim3((unsigned)((parts.rows + per - 1) / per)), kThreads, 0, c.stream, true, 0, g, parts, o, lse);
}

// f(head dimension, type) as constants
template <class F>
int by_type(int d, bool f16, F&& f) {
  using std::integral_constant;
  if (d == 64) return f16 ? f(integral_constant<int, 64>{}, std::true_type{}) : f(integral_constant<int, 64>{}, std::false_type{});
  return f16 ? f(integral_constant<int, 128>{}, std::true_type{}) : f(integral_constant<int, 128>{}, std::false_type{});
}

}  // namespace

int launch_paged_parts(const HostCtx& c, const PagedGeo& g, bool f16, const View& q, const View& k_pages, const View& v_pages,
                       const PartsOut& parts, int most_parts, bool direct, bool clear, const View& o, float* lse) {
  const DecArgs a = {q, o, lse, parts, 0, direct, clear, c.status};
  return by_type(g.d, f16, [&](auto d, auto type) {
    constexpr int D = decltype(d)::value;
    constexpr bool F16 = decltype(type)::value;
    return g.G * g.T > 8 ? launch_parts<D, F16, 2>(c, g, a, k_pages, v_pages, most_parts)
                         : launch_parts<D, F16, 1>(c, g, a, k_pages, v_pages, most_parts);
  });
}

int launch_paged_join(const HostCtx& c, const PagedGeo& g, bool f16, const PartsOut& parts, int most_parts, const View& o, float* lse) {
  return by_type(g.d, f16, [&](auto d, auto type) {
    constexpr int D = decltype(d)::value;
    constexpr bool F16 = decltype(type)::value;
    return most_parts > 8 ? launch_join<D, F16, kWarps>(c, g, parts, o, lse) : launch_join<D, F16, 1>(c, g, parts, o, lse);
  });
}

}  // namespace mosaic
