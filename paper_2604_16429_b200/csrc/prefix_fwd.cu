// Attention of a batch over the prefix that all its members share, on Blackwell tensor cores (tcgen05 + TMEM + TMA).
//
//   s_rj = scale q_r . k_j over all keys of the prefix;  a part of the keys gives every row its maximum m, sum l and sum of e^(s - m) v
// The rows of a key/value head are all members' new tokens and the head's query heads, (b T + i) G + g, so that the prefix is read
// once for the batch and its products are large: tiles of 128 rows, two to a CTA, share every staged tile of 64 keys.  The prefix lies
// in pages of the cache, which a step's boxes fetch one by one.  An item is two tiles and a part of the keys; the join of a row's parts,
// the member's own keys among them, is another kernel's.
//
// Warps (384 threads, persistent, one CTA per SM): 0-3 and 4-7 softmax of tile 0 and 1 (thread = row = TMEM lane; they also bring their
// rows of q, which lie all over the tensor, to shared memory), 8 TMA, 9 and 10 the products of tile 0 and 1.  TMEM as in the
// sliding-window forward: two score buffers of a tile, the 16-bit weights over a buffer's first half, O behind.  Q K^T of a step is issued
// ahead of P V of the step before.  Softmax in base 2; the maximum moves only when it grows by more than 2^8.  Weights round to 16 bits
// once, as operands; the rest is fp32.  Every wait is bounded.
//
// Measured (cycles, 64 members of 4 heads on each of 4 key/value heads of 128, 32768 keys in 37 parts, 148 items of 14 steps): rows of q 5000
// (lane by lane instead of by asynchronous copies 10000), first scores and weights 2000, 1950 a step (what bounds it: window_fwd.cu), sums
// out 4800 (in half lines 6800): 25 us, of which the products at the measured rate would be 10 and the bytes 10.
#include <type_traits>

#include "paged.cuh"

namespace mosaic {

namespace {

constexpr int kThreads = 384;
// Registers a thread: the three warpgroups' shares add up to what the block is launched with, or the increase would wait for good.
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(2 * kSoftmaxRegs + kOtherRegs <= 3 * kLaunchRegs, "the shares exceed the launch's registers");
constexpr uint32_t kTmemCols = 512, kColO = 256;  // scores, and weights over them, below; O of tile t at kColO + d t
constexpr float kRescaleThreshold = 8.0f;         // log2 units: weights stay below 2^8
constexpr int U = 1 << kBoxShift;                 // keys of a step
constexpr int kSlots = 8;                         // ring of key and value tiles
__host__ __device__ constexpr uint32_t score_col(int t, uint32_t b) { return 128 * t + 64 * b; }

template <int D>
struct Smem {
  static constexpr int kTileBytes = kRows * D * 2, kSlotBytes = U * D * 2;
  unsigned char q[2][kTileBytes];
  unsigned char kv[kSlots][kSlotBytes];
  uint4 rows[8][32 * 8];  // a softmax warp's 32 rows of 32 results on their way out
  unsigned long long q_full[2], q_empty[2], kv_full[kSlots], kv_empty[kSlots];
  unsigned long long s_full[2][2], p_full[2][2], pv_done[2][2], drain[2];
  uint32_t tmem_base;
  int abort;
};

struct PrefixArgs {
  View q;
  const int32_t* table;
  PartsOut parts;
  int len, chunk;        // keys of the prefix, of a part (a multiple of U)
  int rows, pairs;       // rows of a key/value head; pairs of tiles
  int box_shift;         // log2 of the rows of a box: a page, at most U
  int box_loads;         // copies that bring a box's channels: with all of a step's rows in one box, one
  int total;             // items
  float inv_g;           // 1 / G
  int* status;
};

// Two tiles of rows and a part of the keys.  Pairs of tiles are neighbours in the list: what they read is the same.
struct Item {
  int hk, part, row0, k0, k1, steps;
  __device__ __forceinline__ void make(const PrefixArgs& a, int index) {
    const int rest = a.pairs == 1 ? index : index / a.pairs, pair = index - rest * a.pairs;
    hk = rest / a.parts.shared;
    part = rest - hk * a.parts.shared;
    row0 = 2 * kRows * pair;
    k0 = part * a.chunk;
    k1 = min(a.len, k0 + a.chunk);
    steps = (k1 - k0 + U - 1) / U;
  }
};

__device__ __forceinline__ int round32(int n) { return (n + 31) & ~31; }

}  // namespace

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    prefix_fwd_kernel(const PagedGeo g, const __grid_constant__ PrefixArgs a, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v) {
  extern __shared__ unsigned char smem_raw[];
  using S = Smem<D>;
  S& sm = *reinterpret_cast<S*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr uint32_t kPart = kRows * 128, kSlotPart = U * 128;  // bytes of a tile's 64 channels
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int* status = a.status;

  if (tid == 0) {
    for (int s = 0; s < kSlots; ++s) { mbar_init(s32(&sm.kv_full[s]), 1); mbar_init(s32(&sm.kv_empty[s]), 2); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s32(&sm.q_full[t]), 128);
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
  // A code is written no earlier than a wait's bound of seconds after its CTA began; the first CTA has cleared the word by then.
  if (blockIdx.x == 0 && tid == 0) status[zero] = 0;
  const uint32_t tmem = cta_tmem_alloc(warp == 9, &sm.tmem_base, kTmemCols);
  volatile int* abort = &sm.abort;
  const int first_item = (int)blockIdx.x + zero;

  if (warp == 8) {
    // ------------------------------------------------------------- TMA producer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    uint32_t slot_no = 0;
    bool ok = true;
    const int boxes = U >> a.box_shift, box = 1 << a.box_shift, in_page = (1 << g.shift) - 1;
    const uint32_t box_bytes = (uint32_t)box * 128;
    // Page numbers of the step's boxes in the lanes, -1 where there is none
    auto look_up = [&](const Item& it, int n) {
      const int key = it.k0 + n * U + (lane % boxes << a.box_shift);
      int id = -1;
      if (lane < boxes * a.box_loads && key < a.len) id = __ldg(a.table + (key >> g.shift));
      return id;
    };
    auto load = [&](const CUtensorMap* map, int ids, int slot, int hk) {
      const uint32_t s = slot_no % kSlots, bar = s32(&sm.kv_full[s]);
      ok = warp_wait_here(s32(&sm.kv_empty[s]), ((slot_no / kSlots) & 1) ^ 1, abort, status);
      if (!ok) return;
      if (lane == 0) mbar_expect_tx(bar, S::kSlotBytes);
      __syncwarp();
      if (lane < boxes * a.box_loads) {  // a lane has a box, or (pages smaller than a step) the half of one
        const int c = lane / boxes, n = lane - c * boxes;
        load_slots(s32(sm.kv[s]) + c * kSlotPart + n * box_bytes, map, bar, (slot + (n << a.box_shift)) & in_page, c, hk,
                   (unsigned)ids < (unsigned)g.pages ? ids : g.pages);  // (rows behind the last page arrive as zeros)
      }
      __syncwarp();
      ++slot_no;
    };
    int index = first_item;
#ifdef MOSAIC_TEST_WITHHOLD_FIRST_LIST
    index = a.total;  // test build only: nothing is ever loaded, so that every wait for it runs out
#endif
    Item it;
    if (index < a.total) it.make(a, index);
    int ids = index < a.total ? look_up(it, 0) : 0, n = 0;
    while (index < a.total && ok) {
      Item after = it;  // the next step's page numbers are asked for ahead
      int next = index, m = n + 1;
      if (m == it.steps) {
        m = 0;
        next += gridDim.x;
        if (next < a.total) after.make(a, next);
      }
      const int ahead = next < a.total ? look_up(after, m) : 0;
      const int slot = it.k0 + n * U;
      load(&map_k, ids, slot, it.hk);
      if (ok) load(&map_v, ids, slot, it.hk);
      it = after;
      index = next;
      n = m;
      ids = ahead;
    }
    // copies must have landed, and their readers be done, before the CTA's memory is released
    const uint32_t first = slot_no > kSlots ? slot_no - kSlots : 0;
    if (lane == 0)
      for (uint32_t s = first; s < slot_no; ++s) {
        if (*abort) mbar_drain(s32(&sm.kv_full[s % kSlots]), (s / kSlots) & 1);
        else wait_here(s32(&sm.kv_empty[s % kSlots]), (s / kSlots) & 1, abort, status);
      }
    __syncwarp();
  } else if (warp == 9 || warp == 10) {
    // ------------------------------------------------------------- products of tile t
    // The whole warp walks the loop, one elected lane issues.  `u` counts the tile's own steps: score buffer u % 2.
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
    int kks = 0, v_there = 0;  // keys of the step in sixteens; rows of the value tile that belong to the prefix
    auto issue_pv = [&]() {    // of step u - 1
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
    for (int index = __shfl_sync(0xffffffffu, first_item, 0); index < a.total && ok; index += gridDim.x) {
      it.make(a, index);
      const bool mine = it.row0 + t * kRows < a.rows;
#pragma unroll 1
      for (int n = 0; n < it.steps; ++n) {
        const uint32_t k_full = s32(&sm.kv_full[2 * pair]), k_empty = s32(&sm.kv_empty[2 * pair]);
        if (!mine) {
          // a tile that does not exist hands its slots on, once they have landed (so never twice in a round)
          if (pending) issue_pv();
          ok = ok && warp_wait_here(k_full, phase, abort, status) && warp_wait_here(k_full + 8, phase, abort, status);
          if (!ok) break;
          if (elect_one()) {
            mbar_arrive(k_empty);
            mbar_arrive(k_empty + 8);
          }
          __syncwarp();
        } else {
          if (n == 0) {  // (a new query tile may be a while: the item before is finished first)
            if (pending) issue_pv();
            ok = ok && warp_wait_here(s32(&sm.q_full[t]), n_q & 1, abort, status);
            ++n_q;
          }
          const int cols = min(U, it.k1 - (it.k0 + n * U));
          const uint32_t id = idesc_n(idesc_qk, round32(cols)), tcs = tmem + score_col(t, u % 2);
          const uint64_t kd = k_ring + (uint64_t)(pair * (kPair >> 4));
          ok = ok && warp_wait_here(k_full, phase, abort, status);
          // P V of the step that had the buffer (two before) reads its weights there: only products of one shape into one accumulator
          // are sure to run in issue order
          if (u >= 2) ok = ok && warp_wait_here(s32(&sm.pv_done[t][u % 2]), (u / 2 - 1) & 1, abort, status);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) umma_ss(tcs, k_major(qd, kk, kPart), k_major(kd, kk, kSlotPart), id, kk > 0);
            tc_commit(s32(&sm.s_full[t][u % 2]));
            tc_commit(k_empty);
            if (n == it.steps - 1) tc_commit(s32(&sm.q_empty[t]));
          }
          __syncwarp();
          if (pending) issue_pv();
          if (!ok) break;
          ++u;
          pending = true;
          fresh = n == 0;
          v_pair = pair;
          v_phase = phase;
          kks = round32(cols) / 16;
          v_there = a.len - (it.k0 + n * U);
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
    // ------------------------------------------------------------- rows of q, softmax of tile t, epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = warp >> 2, row = tid & 127;
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), to = mine + kColO + D * t;
    const uint64_t scale2 = pack2(g.scale_log2, g.scale_log2);
    uint32_t u = 0, n_q = 0;
    bool ok = true;
    Item it;
    for (int index = first_item; index < a.total && ok; index += gridDim.x) {
      it.make(a, index);
      const int r = it.row0 + t * kRows + row;
      if (it.row0 + t * kRows >= a.rows) continue;  // (the whole tile)
      // the row's place: member, token, head
      const int bt = a.rows < (1 << 23) ? quick_div(r, g.G, a.inv_g) : r / g.G, b = g.T == 1 ? bt : bt / g.T;
      const int i = bt - b * g.T, head = it.hk * g.G + r - bt * g.G;
      const bool live = r < a.rows && (!g.q_len || i < __ldg(g.q_len + min(b, g.B - 1)));
      const int at = live ? (b * g.H + head) * g.T + i : -1;
      const bool idle = !__any_sync(0xffffffffu, live);
      // some page of the part is not there: the lanes look at its pages, the first of them while the rows of q are on their way
      const int first_page = it.k0 >> g.shift, pages = ((it.k1 - 1) >> g.shift) - first_page + 1;
      const int probe = __ldg(a.table + first_page + min(lane, pages - 1));
      ok = warp_wait_here(s32(&sm.q_empty[t]), (n_q & 1) ^ 1, abort, status);
      ++n_q;
      if (!ok) break;
      {  // the warp's rows of q, a row or two at a time, whatever their strides; rows that do not exist are zeros
        constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
        const long long src = (long long)b * a.q.sb + head * a.q.sh + i * a.q.sn;
        const uint32_t dst = s32(sm.q[t]);
#pragma unroll
        for (int x = 0; x < kLanes; ++x) {
          const int rr = x * kAtOnce + lane / kLanes, c = lane % kLanes, row_at = (warp & 3) * 32 + rr;
          const long long from = __shfl_sync(0xffffffffu, src, rr);
          const uint32_t bytes = __shfl_sync(0xffffffffu, at, rr) >= 0 ? 16u : 0u;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (c >> 3) * kPart + row_at * 128 + (((c & 7) ^ (row_at & 7)) << 4)),
                       "l"(a.q.data + (bytes ? from + 16 * c : 0)), "r"(bytes)
                       : "memory");
        }
      }
      bool holes = (unsigned)probe >= (unsigned)g.pages;
      for (int page = lane + 32; page < pages; page += 32) holes |= (unsigned)__ldg(a.table + first_page + page) >= (unsigned)g.pages;
      holes = __any_sync(0xffffffffu, holes);
      asm volatile("cp.async.wait_all;\n\tfence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(s32(&sm.q_full[t]));
      float m_ref = -INFINITY, l = 0.f;
      for (int n = 0; n < it.steps; ++n) {
        const int start = it.k0 + n * U, cols = min(U, it.k1 - start);
        const uint32_t b2 = u % 2, ts = mine + score_col(t, b2);
        ok = warp_wait_here(s32(&sm.s_full[t][b2]), (u / 2) & 1, abort, status);
        if (!ok) break;
        ++u;
        if (idle) {  // rows that do not exist: whatever is there serves as weights
          mbar_arrive(s32(&sm.p_full[t][b2]));
          continue;
        }
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
        // weights of 32 keys: the exponentials of eight are under way while the eight before are added up and rounded
        auto weights = [&](const uint32_t (&sc)[32], uint64_t negm2, uint32_t column) {
          uint32_t pk[16];
          float e[4][8];
#pragma unroll
          for (int x = 0; x < 5; ++x) {
            if (x < 4) {
#pragma unroll
              for (int y = 0; y < 8; y += 2) {
                float v, w;
                unpack2(fma2(pack2(__uint_as_float(sc[8 * x + y]), __uint_as_float(sc[8 * x + y + 1])), scale2, negm2), v, w);
                e[x][y] = ex2(v);
                e[x][y + 1] = ex2(w);
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
          float v = max3(__uint_as_float(sc[0]), __uint_as_float(sc[1]), __uint_as_float(sc[2])), w = __uint_as_float(sc[3]);
#pragma unroll
          for (int x = 4; x < 32; x += 4) {
            v = max3(v, __uint_as_float(sc[x]), __uint_as_float(sc[x + 1]));
            w = max3(w, __uint_as_float(sc[x + 2]), __uint_as_float(sc[x + 3]));
          }
          return fmaxf(v, w);
        };
        // What is not there becomes -inf: columns behind the prefix' end, pages outside the pool
        auto mask = [&](int c, uint32_t (&sc)[32]) {
          uint32_t see = low_bits(cols - 32 * c);
          if (holes)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int key = start + 32 * c + 16 * x;
              if (key < it.k1 && (unsigned)__ldg(a.table + (key >> g.shift)) >= (unsigned)g.pages) see &= x ? 0xffffu : 0xffff0000u;
            }
#pragma unroll
          for (int x = 0; x < 32; ++x) sc[x] = (see >> x) & 1u ? sc[x] : 0xff800000u;
        };
        const bool whole = cols == U && !holes;
        if (cols <= 32) {
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
          if (!whole) {
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
          if (n > 0) ok = warp_wait_here(s32(&sm.pv_done[t][b2 ^ 1]), ((u - 2) / 2) & 1, abort, status);  // O is scaled between two products
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
              float v, w;
              unpack2(mul2(pack2(__uint_as_float(ov[x]), __uint_as_float(ov[x + 1])), alpha2), v, w);
              ov[x] = __float_as_uint(v);
              ov[x + 1] = __float_as_uint(w);
            }
            tmem_st32(to + 32 * part, ov);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(s32(&sm.p_full[t][b2]));
      }
      if (!ok) break;
      ok = warp_wait_here(s32(&sm.pv_done[t][(u - 1) % 2]), ((u - 1) / 2) & 1, abort, status);
      if (!ok) break;
      if (idle) continue;
      tc_fence_after();
      // The rows leave by way of shared memory: a warp stores four rows of 128 bytes at a time.
      const long long base = (long long)it.part * a.parts.rows;
      uint4* stage = sm.rows[warp];
#pragma unroll
      for (int part = 0; part < D / 32; ++part) {
        uint32_t ov[32];
        tmem_ld32(to + 32 * part, ov);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 8; ++x) stage[8 * lane + (x ^ (lane & 7))] = make_uint4(ov[4 * x], ov[4 * x + 1], ov[4 * x + 2], ov[4 * x + 3]);
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int rr = 4 * x + (lane >> 3), c = lane & 7, dst = __shfl_sync(0xffffffffu, at, rr);
          const uint4 val = stage[8 * rr + (c ^ (rr & 7))];
          if (dst >= 0) *reinterpret_cast<uint4*>(a.parts.o + (base + dst) * D + 32 * part + 4 * c) = val;
        }
        __syncwarp();
      }
      if (live) a.parts.ml[base + at] = make_float2(m_ref, l);
      tc_fence_before();  // O has been read: the next item's first P V, which waits for these threads' weights, may overwrite it
    }
  }
  cta_tmem_free(warp == 9, tmem, kTmemCols);
}

namespace {
template <int D, bool F16>
int launch(const HostCtx& c, const PagedGeo& g, const PrefixArgs& a, const PoolMaps& maps) {
  // pages smaller than a step come by halves of their channels, which lie a tile's rows apart
  CUtensorMap k = maps.k, v = maps.v;
  if (a.box_loads > 1 && (!make_map_pool(&k, maps.k_pages, D, 1 << g.shift, g.Hkv, g.pages, 1 << a.box_shift, 1) ||
                          !make_map_pool(&v, maps.v_pages, D, 1 << g.shift, g.Hkv, g.pages, 1 << a.box_shift, 1)))
    return MOSAIC_E_CUDA;
  const size_t smem = sizeof(Smem<D>) + 1024;
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup_regs(reinterpret_cast<const void*>(prefix_fwd_kernel<D, F16>), kLaunchRegs, smem, &configured, &sms)) return rc;
  return launch_kernel(prefix_fwd_kernel<D, F16>, dim3((unsigned)(a.total < sms ? a.total : sms)), kThreads, smem, c.stream, true, 0, g, a, k, v);
}

constexpr int pairs_of(long long rows) { return (int)((rows + 2 * kRows - 1) / (2 * kRows)); }
}  // namespace

// Parts of a prefix of `len` keys: as many as make the longest SM's work shortest.  An SM takes ceil(items / SMs) items, each of its part's
// steps and kTurn steps' time for its start and end (measured: 5000 cycles to its rows of q, 2000 to its first weights, 5000 to write
// its sums, against 1970 a step).
constexpr int kTurn = 6;
int prefix_parts(int len, int kv_heads, long long rows, int* chunk) {
  const long long units = (long long)kv_heads * pairs_of(rows);
  const int steps = (len + U - 1) / U;
  long long best = 0;
  int parts = 1;
  for (int n = 1; n <= steps && (n == 1 || units * (n - 1) < 2 * kSms); ++n) {
    const int each = (steps + n - 1) / n;
    if ((steps + each - 1) / each != n) continue;
    const long long cost = (units * n + kSms - 1) / kSms * (each + kTurn);
    if (n == 1 || cost < best) {
      best = cost;
      parts = n;
    }
  }
  *chunk = (steps + parts - 1) / parts * U;
  return parts;
}

int launch_prefix_fwd(const HostCtx& c, const PagedGeo& g, bool f16, const View& q, const PoolMaps& maps, const int32_t* prefix_table,
                      int prefix_len, int chunk, const PartsOut& parts) {
  PrefixArgs a = {};
  a.q = q;
  a.table = prefix_table;
  a.parts = parts;
  a.len = prefix_len;
  a.chunk = chunk;
  const long long rows = (long long)g.B * g.T * g.G;
  a.rows = (int)rows;
  a.inv_g = 1.f / (float)g.G;
  a.pairs = pairs_of(rows);
  a.box_shift = maps.box_shift;
  a.box_loads = a.box_shift < kBoxShift ? g.d / 64 : 1;
  const long long total = (long long)g.Hkv * parts.shared * a.pairs;
  if (total > 0x7ffffff0ll) return MOSAIC_E_UNSUPPORTED;
  a.total = (int)total;
  a.status = c.status;
  if (g.d == 64) return f16 ? launch<64, true>(c, g, a, maps) : launch<64, false>(c, g, a, maps);
  return f16 ? launch<128, true>(c, g, a, maps) : launch<128, false>(c, g, a, maps);
}

}  // namespace mosaic
