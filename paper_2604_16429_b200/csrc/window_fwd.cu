// Forward of the causal sliding-window attention with sinks on Blackwell tensor cores (tcgen05 + TMEM + TMA).
//
//   s_ij = scale q_i . k_j over the keys j that row i sees;  o_i = sum_j exp(s_ij - m_i) v_j / l_i,  lse_i = m_i + log l_i
// in one pass over the keys with a running maximum m and sum l.
//
// A tile is 128 query rows of one head.  The tiles of a key/value head are numbered with the heads of its group fastest, and a
// CTA takes two neighbours: heads of a group read the same keys, so a staged key tile serves 256 rows.  The two tiles walk a
// common sequence of steps of at most 128 keys: the sinks (as many columns as there are, rounded up to 32) unless the window
// still holds them, then the union of the two windows from its first key on; a step that a tile sees nothing of it leaves out.
// Only steps at the window's edges are masked element by element.
//
// Warps (384 threads, persistent, one CTA per SM): 0-3 and 4-7 softmax of tile 0 and 1 (thread = row = TMEM lane), 8 TMA, 9 the
// products of both tiles.  While the softmax warps of one tile work, the tensor core adds P V of the other one and forms its
// next Q K^T.  TMEM (512 columns): S of tile t at 128 t (fp32), P over its first half (16 bit), O at 256 + d t.
// Softmax in base 2 with the scale folded in; the maximum moves (and O is scaled) only when it grows by more than 2^8; a
// quarter of the exponentials run on the FMA pipe, because MUFU gives 16 a clock and SM against 4 d tensor FLOP each.
// Every wait is bounded (status MOSAIC_E_DEVICE_TIMEOUT, copies and products in flight awaited, TMEM freed).
#include <type_traits>

#include "window.cuh"

namespace mosaic {

namespace {

constexpr int kThreads = 384;
// Registers a thread: the softmax threads hold a row of 128 scores.  The three warpgroups' shares add up to what the block is
// launched with (384 threads of 168, which is what the compiler reports), or the increase would wait for good.
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(2 * kSoftmaxRegs + kOtherRegs <= 3 * kLaunchRegs, "the shares exceed the launch's registers");
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;
constexpr float kRescaleThreshold = 8.0f;  // log2 units: P stays below 2^8

template <int D>
struct Smem {
  static constexpr int kTileBytes = kRows * D * 2;
  static constexpr int kSlots = D == 128 ? 5 : 10;  // ring of key and value tiles
  unsigned char q[2][kTileBytes];
  unsigned char kv[kSlots][kTileBytes];
  unsigned long long q_full[2], q_empty[2], kv_full[kSlots], kv_empty[kSlots], s_full[2], p_full[2], o_full[2], drain;
  uint32_t tmem_base;
  int abort;
};

// What a CTA does at a time: two tiles of a key/value head and the keys that they see.
struct Item {
  int b, hk;
  int kl, off, ql;
  int row0[2], head[2];
  int lo[2], hi[2];  // keys of the tile's window (sinks aside); hi <= 0: nothing to compute
  int base, end;     // union of the windows
  int sinks, ns;     // all sinks; those in front of base, which have a step of their own (the others lie in the first of the union)
  int steps;
  __device__ __forceinline__ void make(const WinGeo& g, int per, int index) {
    // the last rows first: in plain causal attention they have the most keys
    const int unit = index % (g.B * g.Hkv), pair = per - 1 - index / (g.B * g.Hkv);
    b = unit / g.Hkv;
    hk = unit - b * g.Hkv;
    const Span s = span_of(g, b);
    kl = s.kl; off = s.off; ql = s.ql;
    base = 0x7fffffff;
    end = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 2 * pair + t, qt = r / g.G;
      row0[t] = qt * kRows;
      head[t] = hk * g.G + (r - qt * g.G);
      const int last = min(row0[t] + kRows, ql) - 1;
      hi[t] = last >= row0[t] ? off + last + 1 : 0;
      lo[t] = max(0, off + row0[t] - g.window + 1);
      if (hi[t] > 0) {
        base = min(base, lo[t]);
        end = max(end, hi[t]);
      }
    }
    sinks = g.sinks;
    ns = end > 0 ? min(sinks, base) : 0;
    steps = end > 0 ? (ns > 0) + (end - base + kRows - 1) / kRows : 0;
  }
  // (selections, so that an item stays in registers)
  __device__ __forceinline__ int lo_of(int t) const { return t ? lo[1] : lo[0]; }
  __device__ __forceinline__ int hi_of(int t) const { return t ? hi[1] : hi[0]; }
  __device__ __forceinline__ int row0_of(int t) const { return t ? row0[1] : row0[0]; }
  __device__ __forceinline__ int head_of(int t) const { return t ? head[1] : head[0]; }
  // keys start .. start + cols - 1 of step n
  __device__ __forceinline__ void step(int n, int& start, int& cols) const {
    const int w = n - (ns > 0);
    start = w < 0 ? 0 : base + w * kRows;
    cols = w < 0 ? ns : min(kRows, end - start);
  }
  __device__ __forceinline__ bool active(int t, int n) const {
    int start, cols;
    step(n, start, cols);
    return hi_of(t) > 0 && (start < sinks || (start < hi_of(t) && start + cols > lo_of(t)));
  }
  // first and last step that tile t takes part in
  __device__ __forceinline__ int first_step(int t) const { return base < sinks || ns > 0 ? 0 : (lo_of(t) - base) / kRows; }
  __device__ __forceinline__ int last_step(int t) const { return (ns > 0) + (hi_of(t) - 1 - base) / kRows; }
};

// All steps of a CTA's items, one after the other
struct Walk {
  Item it;
  int index, n;
  __device__ __forceinline__ bool seek(const WinGeo& g, int per, int total) {  // to the next item that has steps, from `index` on
    for (; index < total; index += gridDim.x) {
      it.make(g, per, index);
      if (it.steps > 0) { n = 0; return true; }
    }
    return false;
  }
  __device__ __forceinline__ bool next(const WinGeo& g, int per, int total) {
    if (++n < it.steps) return true;
    index += gridDim.x;
    return seek(g, per, total);
  }
};

__device__ __forceinline__ int round32(int n) { return (n + 31) & ~31; }

}  // namespace

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    window_fwd_kernel(const WinGeo g, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const Fold fq, const Fold fk, const Fold fv, const View o,
                      float* __restrict__ lse, int* status, int per, int total) {
  extern __shared__ unsigned char smem_raw[];
  using S = Smem<D>;
  S& sm = *reinterpret_cast<S*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr uint32_t kPart = kRows * 128;  // bytes of a tile's 64 channels
  constexpr int kParts = D / 64;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < S::kSlots; ++s) { mbar_init(s32(&sm.kv_full[s]), 1); mbar_init(s32(&sm.kv_empty[s]), 1); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s32(&sm.q_full[t]), 1);
      mbar_init(s32(&sm.q_empty[t]), 1);
      mbar_init(s32(&sm.s_full[t]), 1);
      mbar_init(s32(&sm.p_full[t]), 128);
      mbar_init(s32(&sm.o_full[t]), 1);
    }
    mbar_init(s32(&sm.drain), 1);
    sm.abort = 0;
    cta_publish_barriers();
  }
  const int zero = await_stream();
  // A code is written no earlier than a wait's bound of seconds after its CTA began; the first CTA, which the grid starts with,
  // has cleared the word by then.
  if (blockIdx.x == 0 && tid == 0) status[zero] = 0;
  const uint32_t tmem = cta_tmem_alloc(warp == 9, &sm.tmem_base, kTmemCols);
  volatile int* abort = &sm.abort;

  if (warp == 8) {
    // ------------------------------------------------------------- TMA producer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    uint32_t slot_no = 0, q_no[2] = {0, 0};
    bool ok = true;
    Walk w;
    w.index = (int)blockIdx.x + zero;
#ifdef MOSAIC_TEST_WITHHOLD_FIRST_LIST
    w.index = total;  // test build only: nothing is ever loaded, so that every wait for it runs out
#endif
    if (lane == 0) {
      auto load = [&](const CUtensorMap* map, const Fold& f, int row, int head, int b) {
        const uint32_t s = slot_no % S::kSlots, bar = s32(&sm.kv_full[s]);
        ok = wait_here(s32(&sm.kv_empty[s]), ((slot_no / S::kSlots) & 1) ^ 1, abort, status);
        if (!ok) return;
        mbar_expect_tx(bar, S::kTileBytes);
#pragma unroll
        for (int c = 0; c < kParts; ++c) tma_load_4d(s32(sm.kv[s]) + c * kPart, map, bar, 64 * c, row, head * f.h, b * f.b);
        ++slot_no;
      };
      for (bool more = w.seek(g, per, total); more && ok; more = w.next(g, per, total)) {
        int start, cols;
        w.it.step(w.n, start, cols);
        if (w.n == 0) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || w.it.hi[t] <= 0) continue;
            ok = wait_here(s32(&sm.q_empty[t]), (q_no[t] & 1) ^ 1, abort, status);
            if (!ok) continue;
            mbar_expect_tx(s32(&sm.q_full[t]), S::kTileBytes);
#pragma unroll
            for (int c = 0; c < kParts; ++c)
              tma_load_4d(s32(sm.q[t]) + c * kPart, &map_q, s32(&sm.q_full[t]), 64 * c, w.it.row0[t], w.it.head[t] * fq.h, w.it.b * fq.b);
            ++q_no[t];
          }
        }
        if (ok) load(&map_k, fk, start, w.it.hk, w.it.b);
        if (ok) load(&map_v, fv, start, w.it.hk, w.it.b);
      }
      // copies must have landed, and their readers be done, before the CTA's memory is released
      const uint32_t first = slot_no > S::kSlots ? slot_no - S::kSlots : 0;
      for (uint32_t s = first; s < slot_no; ++s) {
        if (*abort) mbar_drain(s32(&sm.kv_full[s % S::kSlots]), (s / S::kSlots) & 1);
        else wait_here(s32(&sm.kv_empty[s % S::kSlots]), (s / S::kSlots) & 1, abort, status);
      }
      if (*abort)
        for (int t = 0; t < 2; ++t)
          if (q_no[t]) mbar_drain(s32(&sm.q_full[t]), (q_no[t] - 1) & 1);
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------- products of both tiles
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    constexpr uint32_t idesc_qk = make_idesc(false, 0u, F16), idesc_pv = make_idesc(true, (uint32_t)D, F16);
    uint32_t slot_no = 0;            // ring position of the next step's keys
    uint32_t ph_p = 0, ph_q = 0;     // bit t: phase of p_full[t], q_full[t]
    bool ok = true;
    Walk w;
    w.index = (int)blockIdx.x + zero;
    auto wait_kv = [&](uint32_t no) {
      ok = warp_wait_here(s32(&sm.kv_full[no % S::kSlots]), (no / S::kSlots) & 1, abort, status);
    };
    // Tile by tile (runtime t, so that the descriptors of both tiles are not kept at once): P V of the step `cur`, if it has one
    // and the tile takes part, then Q K^T of the step w.n behind it.
    struct Pv { int act, first, last, kks; uint64_t vd; } cur = {0, 0, 0, 0, 0};
    bool more = w.seek(g, per, total), prologue = true;
    while ((more || !prologue) && ok) {
      uint32_t v_no = slot_no - 1;  // the values of `cur` lie between its keys and the next step's
      if (!prologue) {
        int start, cols;
        w.it.step(w.n, start, cols);
        cur.act = cur.first = cur.last = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int on = w.it.active(t, w.n);
          cur.act |= on << t;
          cur.first |= (on && w.n == w.it.first_step(t)) << t;
          cur.last |= (on && w.n == w.it.last_step(t)) << t;
        }
        cur.kks = round32(cols) / 16;
        v_no = slot_no + 1;
        wait_kv(v_no);
        if (!ok) break;
        unsigned char* vt = sm.kv[v_no % S::kSlots];
        if (w.it.kl < g.Nk && start + round32(cols) > w.it.kl) zero_rows<D>(vt, w.it.kl - start, kRows, lane);
        cur.vd = mn_major(s32(vt), kPart);
        more = w.next(g, per, total);
        slot_no += 2;
      }
      if (more) wait_kv(slot_no);
      if (!ok) break;
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        if ((cur.act >> t) & 1) {
          ok = warp_wait_here(s32(&sm.p_full[t]), (ph_p >> t) & 1, abort, status);
          if (!ok) break;
          ph_p ^= 1u << t;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t oc = tmem + kColO + D * t, pc = tmem + kColS + 128 * t, fresh = (cur.first >> t) & 1;
#pragma unroll 2
            for (int kk = 0; kk < cur.kks; ++kk)
              umma_ts(oc, pc + 8 * kk, cur.vd + (uint64_t)((2048 * kk) >> 4), idesc_pv, !fresh || kk > 0);
            if ((cur.last >> t) & 1) tc_commit(s32(&sm.o_full[t]));
          }
          __syncwarp();
        }
        if (more && w.it.active(t, w.n)) {
          if (w.n == w.it.first_step(t)) {
            ok = warp_wait_here(s32(&sm.q_full[t]), (ph_q >> t) & 1, abort, status);
            if (!ok) break;
            ph_q ^= 1u << t;
          }
          int start, cols;
          w.it.step(w.n, start, cols);
          const uint32_t id = idesc_n(idesc_qk, round32(cols));
          const uint64_t qd = smem_desc(s32(sm.q[t])), kd = smem_desc(s32(sm.kv[slot_no % S::kSlots]));
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              umma_ss(tmem + kColS + 128 * t, k_major(qd, kk, kPart), k_major(kd, kk, kPart), id, kk > 0);
            tc_commit(s32(&sm.s_full[t]));
            if (w.n == w.it.last_step(t)) tc_commit(s32(&sm.q_empty[t]));
          }
          __syncwarp();
        }
      }
      if (!ok) break;
      if (elect_one()) {
        if (!prologue) tc_commit(s32(&sm.kv_empty[v_no % S::kSlots]));
        if (more) tc_commit(s32(&sm.kv_empty[slot_no % S::kSlots]));
      }
      __syncwarp();
      prologue = !more;  // (the last pass leaves the loop)
      if (!more) break;
    }
    if (*abort) {  // products already issued must finish before TMEM and shared memory are released
      if (elect_one()) mma_drain(s32(&sm.drain));
      __syncwarp();
    }
  } else if (warp >= 10) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  } else {
    // ------------------------------------------------------------- softmax of tile t, then epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lane_off + kColS + 128 * t, to = tmem + lane_off + kColO + D * t;
    const uint64_t scale2 = pack2(g.scale_log2, g.scale_log2);
    uint32_t n_s = 0, n_o = 0;
    bool ok = true;
    Item it;
    for (int index = (int)blockIdx.x + zero; index < total && ok; index += gridDim.x) {
      it.make(g, per, index);
      const int i = it.row0_of(t) + row, p = it.off + i;
      float m_ref = -INFINITY, l = 0.f;
      const int n1 = it.hi_of(t) > 0 ? it.last_step(t) : -1;
      for (int n = it.hi_of(t) > 0 ? it.first_step(t) : 0; n <= n1; ++n) {
        if (!it.active(t, n)) continue;
        int start, cols;
        it.step(n, start, cols);
        const int chunks = (cols + 31) >> 5;
        // every row of the tile sees every key of the step
        const bool whole = cols == kRows && start + cols <= it.off + it.row0_of(t) + 1 &&
                           (start + cols <= g.sinks || start > it.off + it.row0_of(t) + kRows - 1 - g.window);
        ok = warp_wait_here(s32(&sm.s_full[t]), n_s & 1, abort, status);
        if (!ok) break;
        ++n_s;
        tc_fence_after();
        bool need = false;
        float alpha = 1.f;
        // the step's largest score (scaled): the maximum moves, or stays
        auto move_max = [&](float mx) {
          if (mx > m_ref + kRescaleThreshold || m_ref == -INFINITY) {
            need = m_ref != -INFINITY;
            alpha = need ? ex2(m_ref - mx) : 1.f;
            m_ref = mx;
            l *= alpha;
          }
        };
        uint64_t sum_a = pack2(0.f, 0.f), sum_b = sum_a;
        // P of 32 keys
        auto weights = [&](const uint32_t (&sc)[32], uint64_t negm2, uint32_t column, auto quartic) {
          uint32_t pk[16];
#pragma unroll
          for (int x = 0; x < 32; x += 4) {
            float x0, x1, x2, x3, p2, p3;
            const uint64_t y01 = fma2(pack2(__uint_as_float(sc[x]), __uint_as_float(sc[x + 1])), scale2, negm2);
            const uint64_t y23 = fma2(pack2(__uint_as_float(sc[x + 2]), __uint_as_float(sc[x + 3])), scale2, negm2);
            unpack2(y01, x0, x1);
            unpack2(y23, x2, x3);
            const float p0 = ex2(x0), p1 = ex2(x1);
            if (decltype(quartic)::value && ((x >> 2) & 1)) { ex2_quartic(y23, p2, p3); } else { p2 = ex2(x2); p3 = ex2(x3); }
            sum_a = add2(sum_a, pack2(p0, p1));
            sum_b = add2(sum_b, pack2(p2, p3));
            pk[x >> 1] = pack2<F16>(p0, p1);
            pk[(x >> 1) + 1] = pack2<F16>(p2, p3);
          }
          tmem_st16(column, pk);
        };
        auto largest = [](const uint32_t (&sc)[32]) {
          float a = max3(__uint_as_float(sc[0]), __uint_as_float(sc[1]), __uint_as_float(sc[2])), b = __uint_as_float(sc[3]);
#pragma unroll
          for (int x = 4; x < 32; x += 4) {
            a = max3(a, __uint_as_float(sc[x]), __uint_as_float(sc[x + 1]));
            b = max3(b, __uint_as_float(sc[x + 2]), __uint_as_float(sc[x + 3]));
          }
          return fmaxf(a, b);
        };
        if (whole) {
          uint32_t s0[32], s1[32], s2[32], s3[32];
          tmem_ld32(ts, s0);
          tmem_ld32(ts + 32, s1);
          tmem_ld32(ts + 64, s2);
          tmem_ld32(ts + 96, s3);
          tmem_wait_ld();
          move_max(fmaxf(fmaxf(largest(s0), largest(s1)), fmaxf(largest(s2), largest(s3))) * g.scale_log2);  // scale > 0 commutes with max
          const uint64_t negm2 = pack2(-m_ref, -m_ref);
          weights(s0, negm2, ts, std::true_type{});
          weights(s1, negm2, ts + 16, std::true_type{});
          weights(s2, negm2, ts + 32, std::true_type{});
          weights(s3, negm2, ts + 48, std::true_type{});
        } else {
          // Masked, or fewer than 128 keys: scores are read twice, 32 at a time.  A key that the row does not see weighs exactly
          // zero (the quartic's clamp does not give that).
          const int below = min(p - start + 1, cols), from = p - g.window + 1 - start, sink = g.sinks - start;
          auto masked = [&](int c, uint32_t (&sc)[32]) {
            tmem_ld32(ts + 32 * c, sc);
            tmem_wait_ld();
            const uint32_t see = low_bits(below - 32 * c) & (~low_bits(from - 32 * c) | low_bits(sink - 32 * c));
#pragma unroll
            for (int x = 0; x < 32; ++x) sc[x] = (see >> x) & 1u ? sc[x] : 0xff800000u;
          };
          uint32_t sc[32];
          float mx = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < chunks; ++c) {
            masked(c, sc);
            mx = fmaxf(mx, largest(sc));
          }
          move_max(mx * g.scale_log2);
          const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
          const uint64_t negm2 = pack2(-m_use, -m_use);
#pragma unroll 1
          for (int c = 0; c < chunks; ++c) {
            masked(c, sc);
            weights(sc, negm2, ts + 16 * c, std::false_type{});
          }
        }
        float s0, s1;
        unpack2(add2(sum_a, sum_b), s0, s1);
        l += s0 + s1;
        // (this step's scores are complete, so the previous P V is: one thread issued them in that order)
        if (__any_sync(0xffffffffu, need)) {
          const uint64_t alpha2 = pack2(alpha, alpha);
#pragma unroll 1
          for (int part = 0; part < D / 32; ++part) {
            uint32_t ov[32];
            tmem_ld32(to + 32 * part, ov);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
              float a, b;
              unpack2(mul2(pack2(__uint_as_float(ov[x]), __uint_as_float(ov[x + 1])), alpha2), a, b);
              ov[x] = __float_as_uint(a);
              ov[x + 1] = __float_as_uint(b);
            }
            tmem_st32(to + 32 * part, ov);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(s32(&sm.p_full[t]));
      }
      if (!ok) break;
      const bool live = i < it.ql && (2 * (per - 1 - index / (g.B * g.Hkv)) + t) < g.G * ((g.Nq + kRows - 1) / kRows);
      const float inv = m_ref == -INFINITY ? 0.f : 1.f / l;
      if (n1 >= 0) {
        ok = warp_wait_here(s32(&sm.o_full[t]), n_o & 1, abort, status);
        if (!ok) break;
        ++n_o;
        tc_fence_after();
      }
      char* dst = o.data + it.b * o.sb + it.head_of(t) * o.sh + (long long)i * o.sn;
#pragma unroll 1
      for (int part = 0; part < D / 32; ++part) {
        uint32_t ov[32];
        if (n1 >= 0) {
          tmem_ld32(to + 32 * part, ov);
          tmem_wait_ld();
        }
        if (live) {
          uint4* d4 = reinterpret_cast<uint4*>(dst + 64 * part);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t r[4];
#pragma unroll
            for (int y = 0; y < 4; ++y)
              r[y] = inv != 0.f ? pack2<F16>(__uint_as_float(ov[8 * x + 2 * y]) * inv, __uint_as_float(ov[8 * x + 2 * y + 1]) * inv) : 0u;
            d4[x] = make_uint4(r[0], r[1], r[2], r[3]);
          }
        }
      }
      if (live)
        lse[((long long)it.b * g.H + it.head_of(t)) * g.Nq + i] = m_ref == -INFINITY ? -INFINITY : (m_ref + log2f(l)) * 0.6931471805599453f;
      tc_fence_before();  // O has been read: the next item's first P V, which waits for these threads' P, may overwrite it
    }
  }
  cta_tmem_free(warp == 9, tmem, kTmemCols);
}

namespace {
template <int D, bool F16>
int launch(const HostCtx& c, const WinGeo& g, const View& q, const View& k, const View& v, const View& o, float* lse) {
  CUtensorMap mq, mk, mv;
  if (!make_map_view(&mq, q, D, g.Nq, g.H, g.B, kRows) || !make_map_view(&mk, k, D, g.Nk, g.Hkv, g.B, kRows) ||
      !make_map_view(&mv, v, D, g.Nk, g.Hkv, g.B, kRows))
    return MOSAIC_E_CUDA;
  const size_t smem = sizeof(Smem<D>) + 1024;
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup(reinterpret_cast<const void*>(window_fwd_kernel<D, F16>), smem, &configured, &sms)) return rc;
  const long long tiles = (long long)g.G * ((g.Nq + kRows - 1) / kRows), per = (tiles + 1) / 2, total = per * g.B * g.Hkv;
  if (total > 0x7ffffff0ll) return MOSAIC_E_UNSUPPORTED;
  return launch_kernel(window_fwd_kernel<D, F16>, dim3((unsigned)(total < sms ? total : sms)), kThreads, smem, c.stream, true, 0, g, mq,
                       mk, mv, fold_of(q), fold_of(k), fold_of(v), o, lse, c.status, (int)per, (int)total);
}
}  // namespace

int launch_window_fwd(const HostCtx& c, const WinGeo& g, bool f16, const View& q, const View& k, const View& v, const View& o,
                      float* lse) {
  if (g.d == 64) return f16 ? launch<64, true>(c, g, q, k, v, o, lse) : launch<64, false>(c, g, q, k, v, o, lse);
  return f16 ? launch<128, true>(c, g, q, k, v, o, lse) : launch<128, false>(c, g, q, k, v, o, lse);
}

}  // namespace mosaic
