// Sliding-window attention of one new token per sequence over a cache, linear or rolling.
//
//   o_h = sum_j exp(scale q_h . k_j - m_h) v_j / l_h  over the keys that position k_len - 1 sees
// HBM-bound: the visible keys and values of a key/value head are read once for all query heads of its group (up to 16 at a
// time).  The keys are split over the warps of a CTA and the CTAs of a cluster; every warp keeps a running maximum, sum and
// accumulator of its own, which are joined in a fixed order: the warps' through shared memory, the CTAs' through the cluster's.
//
// A warp takes 16 keys at a time straight into the operands of mma.sync (products of 16 x 8 x 16 are enough here: the tensor
// core's share of a step is a tenth of the loads'), all loads 16 bytes and of whole rows:
//   S^T = K Q^T   (16 keys x 8 heads): a lane's 8 neighbouring channels of a key serve as two contraction steps; which channel
//                 stands at which place of the contraction does not matter as long as Q's operand has the same order
//   O^T += V^T P^T (16 channels x 8 heads): a lane has 8 neighbouring channels of four keys; byte permutes pair up the keys
// P^T turns from an accumulator into an operand by an 8 x 8 transpose within the warp.
//
// Measured (device, window 4096, 16 heads of 128 on 4): 64 members over rolling caches 94 us, 5.0 TB/s; one member 12.0 us, which are
// the latencies of the launch, eight steps a warp and the two joins.  With one CTA for all of a head's keys 81 and 43 us, with four of
// eight warps 93 and 14.5; how many CTAs share a head's keys left to the number of members (with joins whose bits do not depend on it) 105 to
// 178 us for the former.
#include <type_traits>

#include "mma16.cuh"
#include "window.cuh"

namespace mosaic {

namespace {

constexpr int kDecThreads = 128, kDecWarps = kDecThreads / 32;
constexpr int kStepKeys = 16;
constexpr long long kKeysPerCta = 512;

__device__ __forceinline__ uint4 stream_load(const char* p) {  // a cache row is read once
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float cluster_load(const float* mine, uint32_t rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(s32(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

struct DecArgs {
  View q, k, v, o;
  float* lse;
  int ring;      // rolling cache: slots behind the sinks; 0: position = slot
  int head_blocks, ranks;
};

// What warps and CTAs leave for one another
template <int D, int NT>
struct Joint {
  float part_o[kDecWarps][8 * NT][D], part_m[kDecWarps][8 * NT], part_l[kDecWarps][8 * NT];
  float cta_o[8 * NT][D], cta_m[8 * NT], cta_l[8 * NT];
};

// NT: tiles of 8 query heads that a CTA takes
// AHEAD: the next step's rows are asked for before this step's are worked on (the same arithmetic, so the same bits).
template <int D, bool F16, int NT, bool AHEAD>
__global__ void __launch_bounds__(kDecThreads) window_decode_kernel(const WinGeo g, const __grid_constant__ DecArgs a) {
  constexpr int kHeads = 8 * NT;
  extern __shared__ unsigned char smem_raw[];
  Joint<D, NT>& sm = *reinterpret_cast<Joint<D, NT>*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gq = lane >> 2, tq = lane & 3;
  const int ranks = a.ranks, rank = (int)blockIdx.x % ranks;  // (of the cluster)
  const int unit = (int)blockIdx.x / ranks + await_stream(), hb = unit % a.head_blocks, bk = unit / a.head_blocks, b = bk / g.Hkv, hk = bk - b * g.Hkv;
  const int heads = min(kHeads, g.G - hb * kHeads), head0 = hk * g.G + hb * kHeads;

  // visible keys: the sinks, then positions from .. kl - 1
  int kl = g.k_len ? max(__ldg(g.k_len + b), 0) : g.Nk;
  if (!a.ring) kl = min(kl, g.Nk);
  const int ns = min(g.sinks, kl), from = max(kl - g.window, ns), n = ns + kl - from;
  const int turned = a.ring ? (from - ns) % a.ring : from - ns;  // slot of position `from`, counted from the sinks (if any lies there)
  const char* kp = a.k.data + b * a.k.sb + hk * a.k.sh;
  const char* vp = a.v.data + b * a.v.sb + hk * a.v.sh;
  auto slot = [&](int t) {  // of the t-th visible key (clamped to an existing one)
    t = min(t, n - 1);
    int s = t < ns ? t : turned + t;
    if (a.ring && s - ns >= a.ring && t >= ns) s -= a.ring;
    return (long long)s;
  };

  // Q^T operands: head 8 nt + gq, channels 32 c + 8 tq .. + 7
  uint4 qf[NT][D / 32];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      qf[nt][c] = 8 * nt + gq < heads
                      ? __ldg(reinterpret_cast<const uint4*>(a.q.data + b * a.q.sb + (head0 + 8 * nt + gq) * a.q.sh + 64 * c + 16 * tq))
                      : make_uint4(0u, 0u, 0u, 0u);

  float m[NT][2], l[NT][2], acc[NT][D / 16][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[nt][j][0] = acc[nt][j][1] = acc[nt][j][2] = acc[nt][j][3] = 0.f;
  }

  const int stride = ranks * kDecWarps * kStepKeys;
  int t0 = (rank * kDecWarps + warp) * kStepKeys;
  uint4 kn[2][D / 32], vn[4][D / 64];  // a step's rows on their way
  auto fetch = [&](int t) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const char* row = kp + slot(t + gq + 8 * r) * a.k.sn + 16 * tq;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) kn[r][c] = stream_load(row + 64 * c);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {  // keys 2 tq, 2 tq + 1, 2 tq + 8, 2 tq + 9
      const char* row = vp + slot(t + 2 * tq + (r & 1) + 4 * (r & 2)) * a.v.sn + 16 * gq;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) vn[r][c] = stream_load(row + 128 * c);
    }
  };
  if (AHEAD && t0 < n) fetch(t0);
  for (; t0 < n; t0 += stride) {
    if (!AHEAD) fetch(t0);
    uint4 kf[2][D / 32], vf[4][D / 64];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < D / 32; ++c) kf[r][c] = kn[r][c];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) vf[r][c] = vn[r][c];
    if (AHEAD && t0 + stride < n) fetch(t0 + stride);
    uint32_t pt[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};  // (key gq, head 2 tq), (gq, 2 tq + 1), (gq + 8, 2 tq), (gq + 8, 2 tq + 1)
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        mma16816<F16>(s, kf[0][c].x, kf[1][c].x, kf[0][c].y, kf[1][c].y, qf[nt][c].x, qf[nt][c].y);
        mma16816<F16>(s, kf[0][c].z, kf[1][c].z, kf[0][c].w, kf[1][c].w, qf[nt][c].z, qf[nt][c].w);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) s[x] = t0 + gq + 4 * (x & 2) < n ? s[x] * g.scale_log2 : -INFINITY;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float mx = fmaxf(s[x], s[x + 2]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        if (mx > m[nt][x]) {  // (the same in the eight lanes of the head; the first key of a step always exists)
          const float alpha = ex2(m[nt][x] - mx);
          m[nt][x] = mx;
          l[nt][x] *= alpha;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            acc[nt][j][x] *= alpha;
            acc[nt][j][x + 2] *= alpha;
          }
        }
        s[x] = ex2(s[x] - m[nt][x]);
        s[x + 2] = ex2(s[x + 2] - m[nt][x]);
        l[nt][x] += s[x] + s[x + 2];
      }
      pt[nt][0] = transpose8(pack2<F16>(s[0], s[1]));
      pt[nt][1] = transpose8(pack2<F16>(s[2], s[3]));
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const uint32_t w[4][4] = {{vf[0][c].x, vf[0][c].y, vf[0][c].z, vf[0][c].w}, {vf[1][c].x, vf[1][c].y, vf[1][c].z, vf[1][c].w},
                                {vf[2][c].x, vf[2][c].y, vf[2][c].z, vf[2][c].w}, {vf[3][c].x, vf[3][c].y, vf[3][c].z, vf[3][c].w}};
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // rows gq and gq + 8 of the product: channels 64 c + 8 gq + 2 j and the next
        const uint32_t a0 = __byte_perm(w[0][j], w[1][j], 0x5410), a1 = __byte_perm(w[0][j], w[1][j], 0x7632);
        const uint32_t a2 = __byte_perm(w[2][j], w[3][j], 0x5410), a3 = __byte_perm(w[2][j], w[3][j], 0x7632);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma16816<F16>(acc[nt][4 * c + j], a0, a1, a2, a3, pt[nt][0], pt[nt][1]);
      }
    }
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
      for (int j = 0; j < D / 16; ++j)
        *reinterpret_cast<float2*>(&sm.part_o[warp][h][64 * (j >> 2) + 8 * gq + 2 * (j & 3)]) = make_float2(acc[nt][j][x], acc[nt][j][x + 2]);
    }
  __syncthreads();
  for (int e = tid; e < kHeads * D; e += kDecThreads) {
    const int h = e / D, c = e - h * D;
    float mx = -INFINITY, sum = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) mx = fmaxf(mx, sm.part_m[w][h]);
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
      const float f = sm.part_m[w][h] == -INFINITY ? 0.f : ex2(sm.part_m[w][h] - mx);
      sum = fmaf(sm.part_l[w][h], f, sum);
      v = fmaf(sm.part_o[w][h][c], f, v);
    }
    sm.cta_o[h][c] = v;
    if (c == 0) {
      sm.cta_m[h] = mx;
      sm.cta_l[h] = sum;
    }
  }
  cluster_sync();
  // the CTAs' parts: every CTA joins its share of the channels
  const int share = (kHeads * D + ranks - 1) / ranks, e1 = min(kHeads * D, (rank + 1) * share);
  for (int e = rank * share + tid; e < e1; e += kDecThreads) {
    const int h = e / D, c = e - h * D;
    float mx = -INFINITY, sum = 0.f, v = 0.f;
    for (int r = 0; r < ranks; ++r) mx = fmaxf(mx, cluster_load(&sm.cta_m[h], r));
    for (int r = 0; r < ranks; ++r) {
      const float mr = cluster_load(&sm.cta_m[h], r), f = mr == -INFINITY ? 0.f : ex2(mr - mx);
      sum = fmaf(cluster_load(&sm.cta_l[h], r), f, sum);
      v = fmaf(cluster_load(&sm.cta_o[h][c], r), f, v);
    }
    if (h < heads) {
      const uint32_t bits = pack2<F16>(sum > 0.f ? v / sum : sum, 0.f);  // (a sum that is not a number stays one)
      *reinterpret_cast<unsigned short*>(a.o.data + b * a.o.sb + (head0 + h) * a.o.sh + 2 * c) = (unsigned short)bits;
      if (c == 0) a.lse[(long long)b * g.H + head0 + h] = sum > 0.f ? (mx + log2f(sum)) * 0.6931471805599453f : n ? sum : -INFINITY;
    }
  }
  cluster_sync();  // nobody leaves while its part may still be read
}

template <int D, bool F16, int NT, bool AHEAD>
int launch(const HostCtx& c, const WinGeo& g, const DecArgs& a, long long ctas) {
  const size_t smem = sizeof(Joint<D, NT>);
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup(reinterpret_cast<const void*>(window_decode_kernel<D, F16, NT, AHEAD>), smem, &configured, &sms)) return rc;
  return launch_kernel(window_decode_kernel<D, F16, NT, AHEAD>, dim3((unsigned)ctas), kDecThreads, smem, c.stream, true, a.ranks, g, a);
}

// Rows ahead cost registers.  Where they cost no CTA that the SM would need (d = 64 with 8 heads, 4 CTAs an SM; d = 128 with 16, 2 either
// way) they are always taken, elsewhere as long as all CTAs fit two an SM: there the latency of a warp's few steps is all there is.
// Measured with and without (us; caches of 4100 tokens, 4 key/value heads, window 4096, members in front): d = 64, 4 heads a group 1: 10.2
// and 13.0, 32: 30.8 and 38.5; d = 128, 12 a group 1: 15.8 and 18.0, 32: 75 and 83; d = 128, 4 a group 1: 13.3 and 16.0, 8: 17.1 and 19.7,
// but 16: 33.0 and 26.9; d = 64, 12 a group 8: 15.5 and 16.4, but 16: 28.8 and 20.5.
template <int D, bool F16, int NT>
int launch(const HostCtx& c, const WinGeo& g, DecArgs a) {
  int sms = 0;
  if (const int rc = launch_setup(nullptr, 0, nullptr, &sms)) return rc;
  a.head_blocks = (g.G + 8 * NT - 1) / (8 * NT);
  // How many CTAs share a head's keys follows from the most keys that it may have, alone: a unit's bits must not depend on the others.
  const long long keys = (long long)g.window + g.sinks < g.Nk ? (long long)g.window + g.sinks : g.Nk;
  a.ranks = 1;
  while (a.ranks < 8 && keys > a.ranks * kKeysPerCta) a.ranks *= 2;
  const long long ctas = (long long)g.B * g.Hkv * a.head_blocks * a.ranks;
  if (ctas > 0x7fffffffll) return MOSAIC_E_UNSUPPORTED;
  if constexpr ((D == 64) != (NT == 1))
    if (ctas > 2ll * sms) return launch<D, F16, NT, false>(c, g, a, ctas);
  return launch<D, F16, NT, true>(c, g, a, ctas);
}

}  // namespace

int launch_window_decode(const HostCtx& c, const WinGeo& g, bool f16, int ring, const View& q, const View& k, const View& v,
                         const View& o, float* lse) {
  const DecArgs a = {q, k, v, o, lse, ring, 1, 1};
  auto go = [&](auto d, auto type) {
    constexpr int D = decltype(d)::value;
    constexpr bool F16 = decltype(type)::value;
    return g.G > 8 ? launch<D, F16, 2>(c, g, a) : launch<D, F16, 1>(c, g, a);
  };
  using std::integral_constant;
  if (g.d == 64) return f16 ? go(integral_constant<int, 64>{}, std::true_type{}) : go(integral_constant<int, 64>{}, std::false_type{});
  return f16 ? go(integral_constant<int, 128>{}, std::true_type{}) : go(integral_constant<int, 128>{}, std::false_type{});
}

}  // namespace mosaic
