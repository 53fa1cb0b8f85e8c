// Forward of the causal sliding-window attention with sinks on Blackwell tensor cores (tcgen05 + TMEM + TMA).
//
//   s_ij = scale q_i . k_j over the keys j that row i sees;  o_i = sum_j exp(s_ij - m_i) v_j / l_i,  lse_i = m_i + log l_i
// in one pass over the keys with a running maximum m and sum l.
//
// A tile is 128 query rows of one head.  The tiles of a key/value head are numbered with the heads of its group fastest, and a
// CTA takes two neighbours: heads of a group read the same keys, so a staged key tile serves 256 rows.  The two tiles walk a
// common sequence of steps of at most 64 keys: the sinks (as many columns as there are, rounded up to 32), then what else there is in
// the union of the two windows; a step that a tile sees nothing of it leaves out.  The windows' steps of a batch member are cells of
// one grid, so that what a step holds of a row's keys, and with it the bits of the row's results, does not depend on the tile beside
// it.  Only steps at the window's edges are masked element by element.
//
// Warps (384 threads, persistent, one CTA per SM): 0-3 and 4-7 softmax of tile 0 and 1 (thread = row = TMEM lane), 8 TMA, 9 and 10
// the products of tile 0 and 1.  TMEM (512 columns): two score buffers of a tile at 128 t + 64 b (fp32), P over a buffer's first
// half (16 bit), O at 256 + d t.  Q K^T of a step is issued ahead of P V of the step before, so that the tensor core fills one
// buffer while the softmax warps work on the other.  Softmax in base 2 with the scale folded in; the maximum moves (and O is
// scaled) only when it grows by more than 2^8.
// Every wait is bounded (status MOSAIC_E_DEVICE_TIMEOUT, copies and products in flight awaited, TMEM freed).
//
// Bound by the softmax warps and the way round (scores, softmax, P V, the buffer's next scores): a step of 64 keys for both tiles
// takes 1760 cycles at d = 64 and 1970 at d = 128, of which MUFU is busy 1024 (two warps a scheduler), the tensor core 680 and 1310.
// Measured for 8192 tokens, 16 heads of 128 on 4, window 1024 (us): 96, and, before the first rows too had the sinks in a step of their
// own, 95; beside that: the issuing warps finding a step's slots and limits
// anew each time 99; P in columns of its own beside one score buffer, so that no product has to end before the next scores, 101;
// the two tiles taking turns at the exponentials 96 (at d = 64: 6 % slower).  Beside a form of 91 that left out the wait for the
// buffer's earlier product: one warp for both tiles' products 111, 128 keys a step 102, a quarter or an eighth of the exponentials
// on the FMA pipe 101 and 92, a step's two buffers in the hands of two warpgroups each, which pass the running maximum on, 118.
#include <type_traits>

#include "window.cuh"

namespace mosaic {

namespace {

constexpr int kThreads = 384;
// Registers a thread: the softmax threads hold a row's 64 scores of a step.  The three warpgroups' shares add up to what the block is
// launched with (384 threads of 168, which is what the compiler reports), or the increase would wait for good.
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(2 * kSoftmaxRegs + kOtherRegs <= 3 * kLaunchRegs, "the shares exceed the launch's registers");
constexpr uint32_t kTmemCols = 512, kColO = 256;  // S, and P over it, below; O of tile t at kColO + d t
constexpr float kRescaleThreshold = 8.0f;  // log2 units: P stays below 2^8

constexpr int U = 64;          // keys of a step
constexpr int kSlots = 8;      // ring of key and value tiles
__host__ __device__ constexpr uint32_t score_col(int t, uint32_t b) { return 128 * t + 64 * b; }

template <int D>
struct Smem {
  static constexpr int kTileBytes = kRows * D * 2, kSlotBytes = U * D * 2;
  unsigned char q[2][kTileBytes];
  unsigned char kv[kSlots][kSlotBytes];
  uint4 rows[8][32 * 4];  // a softmax warp's 32 rows of 32 results on their way out
  unsigned long long q_full[2], q_empty[2], kv_full[kSlots], kv_empty[kSlots];
  unsigned long long s_full[2][2], p_full[2][2], drain[2];
  unsigned long long pv_done[2][2];  // one a buffer: a thread that has seen a step's scores is at most one phase behind it
  uint32_t tmem_base;
  int abort;
};

// What a CTA does at a time: two tiles of a key/value head and the keys that they see.
struct Item {
  int b, hk;
  int kl, off, ql;
  int row0[2], head[2], tiles;  // tiles: how many of the two there are
  int lo[2], hi[2];  // keys of the tile's window (sinks aside); hi <= 0: nothing to compute
  int base, end;     // union of the windows behind the sinks, from the start of its first cell on (which may be less than 0)
  int sinks, ns;     // sinks (none where every window holds them); those that there are
  int front, steps;  // steps of the sinks, of all
  // UNIFORM: by a whole warp, all of it uniform
  template <bool UNIFORM = false>
  __device__ __forceinline__ void make(const WinGeo& g, int per, int index) {
    // the last rows first: in plain causal attention they have the most keys
    const int unit = index % (g.B * g.Hkv), pair = per - 1 - index / (g.B * g.Hkv);
    b = unit / g.Hkv;
    hk = unit - b * g.Hkv;
    Span s = span_of(g, b);
    if (UNIFORM) {
      s.ql = __shfl_sync(0xffffffffu, s.ql, 0);
      s.kl = __shfl_sync(0xffffffffu, s.kl, 0);
      s.off = s.kl - s.ql;
    }
    kl = s.kl; off = s.off; ql = s.ql;
    base = 0x7fffffff;
    end = 0;
    sinks = kl > g.window ? g.sinks : 0;
    tiles = min(2, g.G * ((g.Nq + kRows - 1) / kRows) - 2 * pair);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 2 * pair + t, qt = r / g.G;
      row0[t] = qt * kRows;
      head[t] = hk * g.G + (r - qt * g.G);
      const int last = min(row0[t] + kRows, ql) - 1;
      hi[t] = last >= row0[t] && t < tiles ? off + last + 1 : 0;
      lo[t] = max(0, off + row0[t] - g.window + 1);
      if (hi[t] > 0) {
        base = min(base, max(lo[t], sinks));
        end = max(end, hi[t]);
      }
    }
    // A full tile's window is window + rows - 1 keys from a key that is `from` modulo U on, and leaves `spare` columns of its last step.
    // Cells at multiples of U cover it with as many steps unless it starts more than that behind one; then, and where more than half of
    // the last step would be left, cells start at the tiles' first keys.  (us with multiples and with first keys, on 4 key heads:
    // 8192 tokens of 16 heads of 128, window 1024, 94.8 and 95.8; 2 x 8192 tokens of 12 heads of 64, window 100, 49.3 and 50.0; 4 x 4096
    // of 16 of 64, window 16, 48.7 and 47.2; chunks of 4 x 1000 rows, 12 heads of 64, window 1000, 50.3 and 48.0.)
    const int from = (off + 1 - g.window) & (U - 1), spare = (1 - g.window - min(ql, kRows)) & (U - 1);
    base -= (base - (kl > g.window && (from > spare || spare >= U / 2) ? from : 0)) & (U - 1);
    ns = min(sinks, end);
    front = (ns + U - 1) / U;
    steps = front + (end > sinks ? (end - base + U - 1) / U : 0);
  }
  // (selections, so that an item stays in registers)
  __device__ __forceinline__ int lo_of(int t) const { return t ? lo[1] : lo[0]; }
  __device__ __forceinline__ int hi_of(int t) const { return t ? hi[1] : hi[0]; }
  __device__ __forceinline__ int row0_of(int t) const { return t ? row0[1] : row0[0]; }
  __device__ __forceinline__ int head_of(int t) const { return t ? head[1] : head[0]; }
  // keys start .. start + cols - 1 of step n
  __device__ __forceinline__ void step(int n, int& start, int& cols) const {
    start = n < front ? n * U : base + (n - front) * U;
    cols = min(U, (n < front ? ns : end) - start);
  }
  // The steps that tile t takes part in: the sinks' in front, and those from first_of(t) to last_of(t)
  __device__ __forceinline__ int first_of(int t) const { return front + (max(lo_of(t), sinks) - base) / U; }
  __device__ __forceinline__ int last_of(int t) const {
    return hi_of(t) > sinks ? front + (hi_of(t) - 1 - base) / U : hi_of(t) > 0 ? front - 1 : -1;
  }
};

// All steps of a CTA's items, one after the other
struct Walk {
  Item it;
  int index, n;
  template <bool UNIFORM = false>
  __device__ __forceinline__ bool seek(const WinGeo& g, int per, int total) {  // to the next item that has steps, from `index` on
    for (; index < total; index += gridDim.x) {
      it.make<UNIFORM>(g, per, index);
      if (it.steps > 0) { n = 0; return true; }
    }
    return false;
  }
  template <bool UNIFORM = false>
  __device__ __forceinline__ bool next(const WinGeo& g, int per, int total) {
    if (++n < it.steps) return true;
    index += gridDim.x;
    return seek<UNIFORM>(g, per, total);
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
  constexpr uint32_t kPart = kRows * 128, kSlotPart = U * 128;  // bytes of a tile's 64 channels
  constexpr int kParts = D / 64;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < kSlots; ++s) { mbar_init(s32(&sm.kv_full[s]), 1); mbar_init(s32(&sm.kv_empty[s]), 2); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s32(&sm.q_full[t]), 1);
      mbar_init(s32(&sm.q_empty[t]), 1);
      for (int b = 0; b < 2; ++b) {
        mbar_init(s32(&sm.s_full[t][b]), 1);
        mbar_init(s32(&sm.p_full[t][b]), 128);
        mbar_init(s32(&sm.pv_done[t][b]), 1);
      }
      mbar_init(s32(&sm.drain[t]), 1);
    }
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
        const uint32_t s = slot_no % kSlots, bar = s32(&sm.kv_full[s]);
        ok = wait_here(s32(&sm.kv_empty[s]), ((slot_no / kSlots) & 1) ^ 1, abort, status);
        if (!ok) return;
        mbar_expect_tx(bar, S::kSlotBytes);
#pragma unroll
        for (int c = 0; c < kParts; ++c) tma_load_4d(s32(sm.kv[s]) + c * kSlotPart, map, bar, 64 * c, row, head * f.h, b * f.b);
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
      const uint32_t first = slot_no > kSlots ? slot_no - kSlots : 0;
      for (uint32_t s = first; s < slot_no; ++s) {
        if (*abort) mbar_drain(s32(&sm.kv_full[s % kSlots]), (s / kSlots) & 1);
        else wait_here(s32(&sm.kv_empty[s % kSlots]), (s / kSlots) & 1, abort, status);
      }
      if (*abort)
        for (int t = 0; t < 2; ++t)
          if (q_no[t]) mbar_drain(s32(&sm.q_full[t]), (q_no[t] - 1) & 1);
    }
  } else if (warp == 9 || warp == 10) {
    // ------------------------------------------------------------- products of tile t
    // The whole warp walks the loop, one elected lane issues; what it walks by is made uniform, so that operands stay in uniform
    // registers.  `u` counts the tile's own steps: score buffer u % 2.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    constexpr uint32_t idesc_qk = make_idesc(false, 0u, F16), idesc_pv = make_idesc(true, (uint32_t)D, F16);
    const int t = warp - 9;
    constexpr uint32_t kPair = 2 * S::kSlotBytes;  // the ring's slots are taken in pairs, a step's keys and its values
    const uint32_t tco = tmem + kColO + D * t;
    const uint64_t qd = smem_desc(s32(sm.q[t])), k_ring = smem_desc(s32(sm.kv[0])), v_ring = mn_major(s32(sm.kv[1]), kSlotPart);
    uint32_t pair = 0, phase = 0, u = 0, n_q = 0;
    bool ok = true;
    // P V of the tile's latest step
    bool pending = false, fresh = false;
    uint32_t v_pair = 0, v_phase = 0;
    int kks = 0, v_there = 0;  // keys of the step in sixteens; rows of the value tile that exist (beyond them it may hold anything)
    auto issue_pv = [&]() {  // of step u - 1
      const uint32_t b = (u - 1) % 2;
      ok = warp_wait_here(s32(&sm.kv_full[2 * v_pair + 1]), v_phase, abort, status);
      if (!ok) return;
      if (v_there < 16 * kks) zero_rows<D>(sm.kv[2 * v_pair + 1], v_there, U, lane);
      const uint64_t vd = v_ring + (uint64_t)(v_pair * (kPair >> 4));
      const uint32_t tcp = tmem + score_col(t, b);
      ok = warp_wait_here(s32(&sm.p_full[t][b]), ((u - 1) / 2) & 1, abort, status);
      if (!ok) return;
      tc_fence_after();
      if (elect_one()) {
        if (kks == U / 16) {
#pragma unroll
          for (int kk = 0; kk < U / 16; ++kk) umma_ts(tco, tcp + 8 * kk, vd + (uint64_t)((2048 * kk) >> 4), idesc_pv, !fresh || kk > 0);
        } else {
#pragma unroll 1
          for (int kk = 0; kk < kks; ++kk) umma_ts(tco, tcp + 8 * kk, vd + (uint64_t)((2048 * kk) >> 4), idesc_pv, !fresh || kk > 0);
        }
        tc_commit(s32(&sm.pv_done[t][b]));
        tc_commit(s32(&sm.kv_empty[2 * v_pair + 1]));
      }
      __syncwarp();
      pending = false;
    };
    Item it;
    for (int index = __shfl_sync(0xffffffffu, (int)blockIdx.x + zero, 0); index < total && ok; index += gridDim.x) {
      it.make<true>(g, per, index);
      const int first = it.first_of(t), last = it.last_of(t), opens = it.front ? 0 : first;
      const bool some_rows = it.kl < g.Nk;  // only then a tile has rows that do not exist
#pragma unroll 1
      for (int n = 0; n < it.steps; ++n) {
        const uint32_t k_full = s32(&sm.kv_full[2 * pair]), k_empty = s32(&sm.kv_empty[2 * pair]);
        if (n > last || (n < first && n >= it.front)) {
          // a tile that leaves a step out hands its slots on, once they have landed (so never twice in a round)
          if (pending) issue_pv();
          ok = ok && warp_wait_here(k_full, phase, abort, status) && warp_wait_here(k_full + 8, phase, abort, status);
          if (!ok) break;
          if (elect_one()) {
            mbar_arrive(k_empty);
            mbar_arrive(k_empty + 8);
          }
          __syncwarp();
        } else {
          if (n == opens) {  // (a new query tile may be a while: the item before is finished first)
            if (pending) issue_pv();
            ok = ok && warp_wait_here(s32(&sm.q_full[t]), n_q & 1, abort, status);
            ++n_q;
          }
          int start, cols;
          it.step(n, start, cols);
          const uint32_t id = idesc_n(idesc_qk, round32(cols)), tcs = tmem + score_col(t, u % 2);
          const uint64_t kd = k_ring + (uint64_t)(pair * (kPair >> 4));
          ok = ok && warp_wait_here(k_full, phase, abort, status);
          // P V of the step that had the buffer (two before) reads its weights there: it was issued before, but only products of
          // one shape into one accumulator are sure to run in issue order.  (The wait costs 8 % at d = 128, nothing at 64.)
          if (u >= 2) ok = ok && warp_wait_here(s32(&sm.pv_done[t][u % 2]), (u / 2 - 1) & 1, abort, status);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) umma_ss(tcs, k_major(qd, kk, kPart), k_major(kd, kk, kSlotPart), id, kk > 0);
            tc_commit(s32(&sm.s_full[t][u % 2]));
            tc_commit(k_empty);
            if (n == last) tc_commit(s32(&sm.q_empty[t]));
          }
          __syncwarp();
          if (pending) issue_pv();
          if (!ok) break;
          ++u;
          pending = true;
          fresh = n == opens;
          v_pair = pair;
          v_phase = phase;
          kks = round32(cols) / 16;
          v_there = some_rows ? it.kl - start : U;
        }
        if (++pair == kSlots / 2) { pair = 0; phase ^= 1; }
      }
    }
    if (ok && pending) issue_pv();
    if (*abort) {  // products already issued must finish before TMEM and shared memory are released
      if (elect_one()) mma_drain(s32(&sm.drain[t]));
      __syncwarp();
    }
  } else if (warp == 11) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  } else {
    // ------------------------------------------------------------- softmax of tile t, then epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = warp >> 2, row = tid & 127;
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), to = mine + kColO + D * t;
    const uint64_t scale2 = pack2(g.scale_log2, g.scale_log2);
    uint32_t u = 0;
    bool ok = true;
    Item it;
    for (int index = (int)blockIdx.x + zero; index < total && ok; index += gridDim.x) {
      it.make(g, per, index);
      const int i = it.row0_of(t) + row, p0 = it.off + it.row0_of(t), p = p0 + row;
      // every row of the tile sees all of a step's U keys if it starts at one of whole0 .. whole1
      const int whole0 = max(p0 + kRows - g.window, it.sinks), whole1 = p0 + 1 - U;
      const int window = max(p + 1 - g.window, it.sinks);  // the row's first key behind the sinks
      float m_ref = -INFINITY, l = 0.f;
      const int last = it.last_of(t), first = it.first_of(t);
      const int front = it.front, steps = last < 0 ? 0 : front + max(last + 1 - first, 0), window0 = it.base + (first - 2 * front) * U;
      for (int n = 0; n < steps; ++n) {
        const int start = n < front ? n * U : window0 + n * U, cols = min(U, (n < front ? it.ns : it.end) - start);
        const uint32_t b = u % 2, ts = mine + score_col(t, b);
        ok = warp_wait_here(s32(&sm.s_full[t][b]), (u / 2) & 1, abort, status);
        if (!ok) break;
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
        // P of 32 keys: the exponentials of eight are under way while the eight before are added up and rounded
        auto weights = [&](const uint32_t (&sc)[32], uint64_t negm2, uint32_t column) {
          uint32_t pk[16];
          float e[4][8];
#pragma unroll
          for (int x = 0; x < 5; ++x) {
            if (x < 4) {
#pragma unroll
              for (int y = 0; y < 8; y += 2) {
                float a, c;
                unpack2(fma2(pack2(__uint_as_float(sc[8 * x + y]), __uint_as_float(sc[8 * x + y + 1])), scale2, negm2), a, c);
                e[x][y] = ex2(a);
                e[x][y + 1] = ex2(c);
              }
            }
            if (x > 0) {
#pragma unroll
              for (int y = 0; y < 8; y += 4) {
                sum_a = add2(sum_a, pack2(e[x - 1][y], e[x - 1][y + 1]));
                sum_b = add2(sum_b, pack2(e[x - 1][y + 2], e[x - 1][y + 3]));
                pk[(8 * (x - 1) + y) >> 1] = pack2<F16>(e[x - 1][y], e[x - 1][y + 1]);
                pk[((8 * (x - 1) + y) >> 1) + 1] = pack2<F16>(e[x - 1][y + 2], e[x - 1][y + 3]);
              }
            }
          }
          tmem_st16(column, pk);
        };
        auto largest = [](const uint32_t (&sc)[32]) {
          float a = max3(__uint_as_float(sc[0]), __uint_as_float(sc[1]), __uint_as_float(sc[2])), c = __uint_as_float(sc[3]);
#pragma unroll
          for (int x = 4; x < 32; x += 4) {
            a = max3(a, __uint_as_float(sc[x]), __uint_as_float(sc[x + 1]));
            c = max3(c, __uint_as_float(sc[x + 2]), __uint_as_float(sc[x + 3]));
          }
          return fmaxf(a, c);
        };
        // What the row does not see becomes -inf.  On an edge most groups of 32 keys are seen by all rows of the warp.
        auto mask = [&](int c, uint32_t (&sc)[32]) {
          const int at = start + 32 * c;
          const uint32_t see = low_bits(min(p + 1 - at, cols - 32 * c)) & ~low_bits((n < front ? 0 : window) - at);
          if (__all_sync(0xffffffffu, see == 0xffffffffu)) return;
#pragma unroll
          for (int x = 0; x < 32; ++x) sc[x] = (see >> x) & 1u ? sc[x] : 0xff800000u;
        };
        if (cols <= 32) {  // the sinks, or the end of a chunk
          uint32_t sc[32];
          tmem_ld32(ts, sc);
          tmem_wait_ld();
          mask(0, sc);
          move_max(largest(sc) * g.scale_log2);
          const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
          weights(sc, pack2(-m_use, -m_use), ts);
        } else {
          uint32_t s0[32], s1[32];
          tmem_ld32(ts, s0);
          tmem_ld32(ts + 32, s1);
          tmem_wait_ld();
          if (start < whole0 || start > whole1) {
            mask(0, s0);
            mask(1, s1);
          }
          move_max(fmaxf(largest(s0), largest(s1)) * g.scale_log2);  // scale > 0 commutes with max
          const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
          const uint64_t negm2 = pack2(-m_use, -m_use);
          weights(s0, negm2, ts);
          weights(s1, negm2, ts + 16);
        }
        float la, lb;
        unpack2(add2(sum_a, sum_b), la, lb);
        l += la + lb;
        if (__any_sync(0xffffffffu, need)) {
          if (u > 0) ok = warp_wait_here(s32(&sm.pv_done[t][b ^ 1]), ((u - 1) / 2) & 1, abort, status);  // O is scaled between two products
          if (!ok) break;
          tc_fence_after();
          const uint64_t alpha2 = pack2(alpha, alpha);
#pragma unroll 1
          for (int part = 0; part < D / 32; ++part) {
            uint32_t ov[32];
            tmem_ld32(to + 32 * part, ov);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
              float a, c;
              unpack2(mul2(pack2(__uint_as_float(ov[x]), __uint_as_float(ov[x + 1])), alpha2), a, c);
              ov[x] = __float_as_uint(a);
              ov[x + 1] = __float_as_uint(c);
            }
            tmem_st32(to + 32 * part, ov);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(s32(&sm.p_full[t][b]));
        ++u;
      }
      if (!ok) break;
      const bool live = i < it.ql && t < it.tiles;
      const float inv = m_ref == -INFINITY ? 0.f : 1.f / l;
      if (last >= 0) {
        ok = warp_wait_here(s32(&sm.pv_done[t][(u - 1) % 2]), ((u - 1) / 2) & 1, abort, status);
        if (!ok) break;
        tc_fence_after();
      }
      // The rows leave by way of shared memory: a warp stores eight rows of 64 bytes at a time.  (Every thread its own row: 32
      // lines an instruction.)
      const unsigned there = __ballot_sync(0xffffffffu, live);
      char* dst = o.data + it.b * o.sb + it.head_of(t) * o.sh + (long long)(it.row0_of(t) + (row & ~31)) * o.sn;
      uint4* stage = sm.rows[warp];
#pragma unroll 1
      for (int part = 0; part < D / 32; ++part) {
        uint32_t ov[32];
        if (last >= 0) {
          tmem_ld32(to + 32 * part, ov);
          tmem_wait_ld();
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          uint32_t r[4];
#pragma unroll
          for (int y = 0; y < 4; ++y)
            r[y] = inv != 0.f ? pack2<F16>(__uint_as_float(ov[8 * x + 2 * y]) * inv, __uint_as_float(ov[8 * x + 2 * y + 1]) * inv) : 0u;
          stage[4 * lane + (x ^ ((lane >> 1) & 3))] = make_uint4(r[0], r[1], r[2], r[3]);
        }
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int rr = 8 * x + (lane >> 2), c = lane & 3;
          const uint4 val = stage[4 * rr + (c ^ ((rr >> 1) & 3))];
          if ((there >> rr) & 1u) *reinterpret_cast<uint4*>(dst + rr * o.sn + 64 * part + 16 * c) = val;
        }
        __syncwarp();
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
  if (!make_map_view(&mq, q, D, g.Nq, g.H, g.B, kRows) || !make_map_view(&mk, k, D, g.Nk, g.Hkv, g.B, U) ||
      !make_map_view(&mv, v, D, g.Nk, g.Hkv, g.B, U))
    return MOSAIC_E_CUDA;
  const size_t smem = sizeof(Smem<D>) + 1024;
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup_regs(reinterpret_cast<const void*>(window_fwd_kernel<D, F16>), kLaunchRegs, smem, &configured, &sms)) return rc;
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
