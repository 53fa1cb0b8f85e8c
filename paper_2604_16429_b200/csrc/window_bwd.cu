// Backward of the causal sliding-window attention with sinks on Blackwell tensor cores (tcgen05 + TMEM + TMA).
//
//   P_ij = exp(s_ij - lse_i), dP_ij = dO_i . v_j, D_i = dO_i . O_i, dS_ij = P_ij (dP_ij - D_i)
//   dq_i = scale sum_j dS_ij k_j;  dk_j = scale sum_i dS_ij q_i;  dv_j = sum_i P_ij dO_i
//
// Two passes of one kernel, each with the tile that it writes resident and the other side streaming by in chunks of 64 rows, so
// that every sum has one owner and a fixed order (no atomics):
//   query-stationary  tile = 128 query rows (Q, dO); chunks of K and V: the sinks in front of the window, then the window
//   key-stationary    tile = 128 keys (K, V); chunks of Q and dO of every head of the group, the rows whose window holds a key of
//                     the tile.  The sinks' keys have all later rows besides; these are cut into pieces as long as a tile's own
//                     list, items of their own whose sums (fp32) a last kernel adds in order.
// Per chunk the first product pair is S and dP (key-stationary: their transposes), then the row threads (thread = row of the tile
// = TMEM lane) form P and dS in 16 bits in the place of S and dP, operands from tensor memory of the sums' products.  As many chunk
// buffers as groups of row threads (three; two where the sums of d = 128 leave no more tensor memory): while the groups work on
// their chunks the tensor core adds an earlier one's sums and forms a later one's S and dP.  TMEM (512 columns): S, dP of buffer b
// at 128 b and 128 b + 64 (P and dS of rows 0 to 31 of the chunk in the first half of either, of the others in the second), behind
// them dS x, then P^T y.
// Rounded to 16 bits: P and dS as operands (the tensor core takes no wider ones; it makes the gradients' error 1.4 times that of
// results rounded once), the results.  Items with the sinks' keys add what those roundings left off in a second product, so that the
// few largest gradients, sums over all rows, are as exact as results rounded once (error over the sinks' keys 0.0023 -> 0.0017 of their
// size in bf16; 4 % of a training pass of 49152 tokens with window 2048, 7 % of 4096 with window 1024, in which is what the operands'
// registers cost: the key-stationary kernel of d = 64 spills 84 bytes a thread in bf16 instead of 28).  Every wait is bounded.
//
// Bound by the way round a chunk's buffer (products, row threads, sums, and their hand-offs) and by the issuing warps: a chunk takes
// about 900 cycles at d = 64 where MUFU needs 512 and the tensor core 540 (query-stationary) or 680, and of that an issuing warp's
// own instructions 600 to 800.  Measured for both passes (us, 37 heads of 4608 tokens, window 3968: query-, key-stationary): this
// form, without sinks, 225, 264 at d = 64 and 326, 449 at d = 128; one warp issuing S and dP of the query-stationary pass 241 and 367, two in the
// key-stationary 275 and 479; slots and limits found anew for each chunk 234, 275 and 335, 473 (with one warp 262, 264 and 380, 468);
// P and dS in columns of their own, two groups 229, 284 and 364, 491; the two sums from a warp each 232, 270 and 330, 455; a part of
// the exponentials on the FMA pipe changed nothing, nor did a second pair of resident tiles for the next item (d = 64: 223, 264).
#include <type_traits>

#include "window.cuh"

namespace mosaic {

namespace {

constexpr int kChunkRows = 64;
constexpr uint32_t kTmemCols = 512;

// Groups of row threads, each with a chunk buffer: three, where tensor memory holds three beside the sums.
template <int D, bool KEYS>
struct Plan {
  static constexpr int kGroups = KEYS && D == 128 ? 2 : 3;
  static constexpr uint32_t kColAcc = 128 * kGroups;
  static constexpr int kWTma = 4 * kGroups, kWMma = kWTma + 1, kThreads = 128 * (kGroups + 1);
  static constexpr int kIssuers = KEYS ? 1 : 2;  // warps that issue S and dP, of every other chunk each
  // Registers a thread: the warpgroups' shares add up to what the block is launched with (which is what the compiler reports), or
  // the increase would wait for good.
  static constexpr int kLaunchRegs = kGroups == 2 ? 168 : 128, kRowRegs = kGroups == 2 ? 208 : 144, kOtherRegs = kGroups == 2 ? 88 : 80;
  static_assert(kGroups * kRowRegs + kOtherRegs <= (kGroups + 1) * kLaunchRegs, "the shares exceed the launch's registers");
  static_assert(kColAcc + (KEYS ? 2 * D : D) <= kTmemCols, "tensor memory");
};

template <int D>
struct Smem {
  static constexpr int kTileBytes = kRows * D * 2, kChunkBytes = kChunkRows * D * 2;
  static constexpr int kSlots = D == 128 ? 4 : 8;
  struct Slot {
    unsigned char x[kChunkBytes], y[kChunkBytes];
  };
  unsigned char x0[kTileBytes], y0[kTileBytes];  // the resident tiles
  Slot ring[kSlots];
  float stat[kSlots][2][kChunkRows];             // key-stationary: -lse (base 2) and -D of the chunk's rows
  unsigned long long st_full, st_empty, ring_full[kSlots], ring_empty[kSlots], sd_full[3], p_full[3], added[3], acc_full, acc_free, drain[3];
  uint32_t tmem_base;
  int abort;
};

struct BwdArgs {
  View dx0, dy0;                  // dq; or dk, dv
  const float *neg_lse2, *neg_d;  // [B, H, pad]
  float* partial;                 // [B, Hkv, pieces + 1, 2, sinks, d]
  int pad, tiles, pieces;         // tiles and sink pieces of a unit
  int piece_rows;
};

// Rows of the sinks' keys beyond the window of tile 0: its own list ends at row `end`, in whole chunks
__device__ __forceinline__ int first_tile_end(const WinGeo& g, const Span& s) {
  const int first = max(0, -s.off) / kChunkRows * kChunkRows, e = min(s.ql, kRows - 1 + g.window - s.off);
  return e > first ? first + (e - first + kChunkRows - 1) / kChunkRows * kChunkRows : first;
}

// What two numbers have beyond their 16-bit roundings, in 16 bits
template <bool F16>
__device__ __forceinline__ uint32_t rest(float a, float b, uint32_t rounded) {
  float ra, rb;
  unpack16x2(rounded, F16, ra, rb);
  return pack2<F16>(a - ra, b - rb);
}

template <bool KEYS>
struct Item {
  int b, hk, head, piece, row0, rows;  // rows: of the tile that exist
  int off, ql, kl;
  int per, chunks;          // chunks of a head, of all
  int front, base, end, ns; // query-stationary: chunks of sinks in front, then keys base .. end - 1; key-stationary: rows base .. end - 1
  template <bool UNIFORM = false>  // by a whole warp, all of it uniform
  __device__ __forceinline__ void make(const WinGeo& g, const BwdArgs& a, int index) {
    const int heads = KEYS ? g.Hkv : g.H;
    const int unit = index % (g.B * heads), i = index / (g.B * heads);
    b = unit / heads;
    head = unit - b * heads;
    hk = KEYS ? head : head / g.G;
    Span s = span_of(g, b);
    if (UNIFORM) {
      s.ql = __shfl_sync(0xffffffffu, s.ql, 0);
      s.kl = __shfl_sync(0xffffffffu, s.kl, 0);
      s.off = s.kl - s.ql;
    }
    off = s.off; ql = s.ql; kl = s.kl;
    front = ns = 0;
    if constexpr (KEYS) {
      head = hk * g.G;
      piece = max(0, i - a.tiles + 1);
      row0 = piece ? 0 : i * kRows;
      rows = min(kRows, kl - row0);
      if (piece == 0) {
        base = max(0, row0 - off) / kChunkRows * kChunkRows;
        end = min(ql, row0 + kRows - 1 + g.window - off);
      } else {
        base = first_tile_end(g, s) + (piece - 1) * a.piece_rows;
        end = min(ql, base + a.piece_rows);
      }
      per = rows > 0 && end > base ? (end - base + kChunkRows - 1) / kChunkRows : 0;
      chunks = per * g.G;
    } else {
      piece = 0;
      row0 = (a.tiles - 1 - i) * kRows;  // the last rows first: in plain causal attention they have the most keys
      rows = min(kRows, ql - row0);
      base = max(0, off + row0 - g.window + 1);
      end = off + min(row0 + kRows, ql);
      ns = min(g.sinks, base);
      front = (ns + kChunkRows - 1) / kChunkRows;
      per = chunks = rows > 0 && end > 0 ? front + (end - base + kChunkRows - 1) / kChunkRows : 0;
    }
  }
  // Key-stationary: the sinks' keys are in the tile, whose gradients are sums over all rows and the largest there are.
  __device__ __forceinline__ bool holds_sinks(const WinGeo& g) const { return row0 == 0 && g.sinks > 0; }
  // first row and number of rows of chunk n of a head
  __device__ __forceinline__ void chunk(int n, int& start, int& cols) const {
    start = !KEYS && n < front ? n * kChunkRows : base + (n - (KEYS ? 0 : front)) * kChunkRows;
    cols = min(kChunkRows, (KEYS ? ql : n < front ? ns : end) - start);
  }
};

}  // namespace

template <int D, bool F16, bool KEYS>
__global__ void __launch_bounds__(Plan<D, KEYS>::kThreads, 1)
    window_bwd_kernel(const WinGeo g, const __grid_constant__ CUtensorMap map_x0, const __grid_constant__ CUtensorMap map_y0,
                      const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_y, const Fold fx0,
                      const Fold fy0, const Fold fx, const Fold fy, const __grid_constant__ BwdArgs a, int* status, int total) {
  extern __shared__ unsigned char smem_raw[];
  using S = Smem<D>;
  using P = Plan<D, KEYS>;
  constexpr int kGroups = P::kGroups;
  constexpr uint32_t kColAcc = P::kColAcc;
  S& sm = *reinterpret_cast<S*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr uint32_t kPart = kRows * 128, kChunkPart = kChunkRows * 128;
  constexpr int kParts = D / 64;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    mbar_init(s32(&sm.st_full), 1);
    mbar_init(s32(&sm.st_empty), P::kIssuers);
    for (int s = 0; s < S::kSlots; ++s) { mbar_init(s32(&sm.ring_full[s]), 1); mbar_init(s32(&sm.ring_empty[s]), 1); }
    for (int i = 0; i < kGroups; ++i) { mbar_init(s32(&sm.sd_full[i]), 1); mbar_init(s32(&sm.p_full[i]), 128); mbar_init(s32(&sm.added[i]), 1); }
    mbar_init(s32(&sm.acc_full), 1);
    mbar_init(s32(&sm.acc_free), 256);
    mbar_init(s32(&sm.drain[0]), 1);
    mbar_init(s32(&sm.drain[1]), 1);
    mbar_init(s32(&sm.drain[2]), 1);
    sm.abort = 0;
    cta_publish_barriers();
  }
  const int first_item = (int)blockIdx.x + await_stream();
  const uint32_t tmem = cta_tmem_alloc(warp == P::kWMma, &sm.tmem_base, kTmemCols);
  volatile int* abort = &sm.abort;
  Item<KEYS> it;

  if (warp == P::kWTma) {
    // ------------------------------------------------------------- TMA producer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kOtherRegs));
    if (lane == 0) {
      uint32_t cc = 0, items = 0;
      bool ok = true;
#ifdef MOSAIC_TEST_WITHHOLD_FIRST_LIST
      total = 0;  // test build only: nothing is ever loaded
#endif
      for (int index = first_item; index < total && ok; index += gridDim.x) {
        it.make(g, a, index);
        if (it.chunks == 0) continue;
        ok = wait_here(s32(&sm.st_empty), (items & 1) ^ 1, abort, status);
        if (!ok) break;
        mbar_expect_tx(s32(&sm.st_full), 2 * S::kTileBytes);
#pragma unroll
        for (int c = 0; c < kParts; ++c) {
          tma_load_4d(s32(sm.x0) + c * kPart, &map_x0, s32(&sm.st_full), 64 * c, it.row0, (KEYS ? it.hk : it.head) * fx0.h, it.b * fx0.b);
          tma_load_4d(s32(sm.y0) + c * kPart, &map_y0, s32(&sm.st_full), 64 * c, it.row0, (KEYS ? it.hk : it.head) * fy0.h, it.b * fy0.b);
        }
        ++items;
        int h = KEYS ? it.head : it.hk;
        for (int n = 0, j = 0; n < it.chunks; ++n, ++cc) {
          const uint32_t s = cc % S::kSlots, bar = s32(&sm.ring_full[s]);
          ok = wait_here(s32(&sm.ring_empty[s]), ((cc / S::kSlots) & 1) ^ 1, abort, status);
          if (!ok) break;
          int start, cols;
          it.chunk(j, start, cols);
          mbar_expect_tx(bar, 2 * S::kChunkBytes + (KEYS ? 2 * kChunkRows * 4 : 0));
#pragma unroll
          for (int c = 0; c < kParts; ++c) {
            tma_load_4d(s32(sm.ring[s].x) + c * kChunkPart, &map_x, bar, 64 * c, start, h * fx.h, it.b * fx.b);
            tma_load_4d(s32(sm.ring[s].y) + c * kChunkPart, &map_y, bar, 64 * c, start, h * fy.h, it.b * fy.b);
          }
          if constexpr (KEYS) {
            const long long at = ((long long)it.b * g.H + h) * a.pad + start;  // start is a multiple of 64
            bulk_load(s32(sm.stat[s][0]), a.neg_lse2 + at, kChunkRows * 4, bar);
            bulk_load(s32(sm.stat[s][1]), a.neg_d + at, kChunkRows * 4, bar);
          }
          if (++j == it.per) { j = 0; ++h; }
        }
      }
      // copies must have landed, and their readers be done, before the CTA's memory is released
      const uint32_t first = cc > S::kSlots ? cc - S::kSlots : 0;
      for (uint32_t s = first; s < cc; ++s) {
        if (*abort) mbar_drain(s32(&sm.ring_full[s % S::kSlots]), (s / S::kSlots) & 1);
        else wait_here(s32(&sm.ring_empty[s % S::kSlots]), (s / S::kSlots) & 1, abort, status);
      }
      if (*abort && items) mbar_drain(s32(&sm.st_full), (items - 1) & 1);
    }
  } else if (warp == P::kWMma || (P::kIssuers == 2 && warp == P::kWMma + 2)) {
    // ------------------------------------------------------------- S and dP
    // (The whole warp walks the loop, one elected lane issues; what it walks by is uniform, so that operands stay in uniform registers.)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kOtherRegs));
    constexpr uint32_t idesc = make_idesc(false, 64u, F16), kStep = P::kIssuers;
    const uint32_t mine = P::kIssuers == 1 || warp == P::kWMma ? 0u : 1u;
    const uint64_t x0d = smem_desc(s32(sm.x0)), y0d = smem_desc(s32(sm.y0)), ring = smem_desc(s32(sm.ring));
    uint32_t s = mine, buf = mine, ring_phase = 0, buf_phase = 0, items = 0;
    int n = (int)mine;
    bool ok = true;
    for (int index = __shfl_sync(0xffffffffu, first_item, 0); index < total && ok; index += gridDim.x) {
      it.template make<true>(g, a, index);
      if (it.chunks == 0) continue;
      ok = warp_wait_here(s32(&sm.st_full), items & 1, abort, status);
      ++items;
      if (n >= it.chunks && elect_one()) mbar_arrive(s32(&sm.st_empty));
      __syncwarp();
      int j = KEYS ? n % it.per : n;
#pragma unroll 1
      for (; n < it.chunks && ok; n += kStep) {
        ok = warp_wait_here(s32(&sm.ring_full[s]), ring_phase, abort, status);
        // the sums of the chunk that had the buffer read its P and dS there (products of different shapes are not ordered by being
        // issued in order)
        ok = ok && warp_wait_here(s32(&sm.added[buf]), buf_phase ^ 1, abort, status);
        if (!ok) break;
        // (of the rows of a chunk only a list's last ones may not exist)
        if (j == it.per - 1 || (!KEYS && j < it.front)) {
          int start, cols;
          it.chunk(j, start, cols);
          const int there = (KEYS ? it.ql : it.kl) - start;  // rows of the chunk that exist
          if (there < kChunkRows && start + there < (KEYS ? g.Nq : g.Nk)) {
            zero_rows<D>(sm.ring[s].x, there, kChunkRows, lane);
            if constexpr (KEYS) zero_rows<D>(sm.ring[s].y, there, kChunkRows, lane);
          }
        }
        j += kStep;
        if (KEYS && j >= it.per) j = kStep == 1 ? 0 : j % it.per;
        tc_fence_after();
        const uint64_t xd = ring + (uint64_t)(s * (uint32_t)(sizeof(typename S::Slot) >> 4)), yd = xd + (S::kChunkBytes >> 4);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            umma_ss(tmem + 128 * buf, k_major(x0d, kk, kPart), k_major(xd, kk, kChunkPart), idesc, kk > 0);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            umma_ss(tmem + 128 * buf + 64, k_major(y0d, kk, kPart), k_major(yd, kk, kChunkPart), idesc, kk > 0);
          tc_commit(s32(&sm.sd_full[buf]));
          if (n >= it.chunks - (int)kStep) tc_commit(s32(&sm.st_empty));
        }
        __syncwarp();
        if ((s += kStep) >= (uint32_t)S::kSlots) { s -= S::kSlots; ring_phase ^= 1; }
        if ((buf += kStep) >= (uint32_t)kGroups) { buf -= kGroups; buf_phase ^= 1; }
      }
      n -= it.chunks;
    }
    if (*abort) {
      if (elect_one()) mma_drain(s32(&sm.drain[2 * mine]));
      __syncwarp();
    }
  } else if (warp == P::kWMma + 1) {
    // ------------------------------------------------------------- sums: dS x, and P^T y
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kOtherRegs));
    constexpr uint32_t idesc = make_idesc(true, (uint32_t)D, F16);
    const uint64_t ring = mn_major(s32(sm.ring), kChunkPart);
    auto add = [&](uint32_t acc, uint32_t weights, uint64_t rows, bool more) {
#pragma unroll
      for (int kk = 0; kk < kChunkRows / 16; ++kk)
        umma_ts(acc, weights + 32 * (kk >> 1) + 8 * (kk & 1), rows + (uint64_t)((2048 * kk) >> 4), idesc, more || kk > 0);
    };
    uint32_t s = 0, buf = 0, buf_phase = 0, items = 0;
    bool ok = true;
    for (int index = __shfl_sync(0xffffffffu, first_item, 0); index < total && ok; index += gridDim.x) {
      it.template make<true>(g, a, index);
      if (it.chunks == 0) continue;
      const bool fine = KEYS && it.holds_sinks(g);
      if (items > 0) ok = warp_wait_here(s32(&sm.acc_free), (items - 1) & 1, abort, status);  // the item before has been read
      ++items;
#pragma unroll 1
      for (int n = 0; n < it.chunks && ok; ++n) {
        ok = warp_wait_here(s32(&sm.p_full[buf]), buf_phase, abort, status);
        if (!ok) break;
        tc_fence_after();
        const uint64_t xd = ring + (uint64_t)(s * (uint32_t)(sizeof(typename S::Slot) >> 4)), yd = xd + (S::kChunkBytes >> 4);
        if (elect_one()) {
          if constexpr (KEYS) add(tmem + kColAcc + D, tmem + 128 * buf, yd, n > 0);
          add(tmem + kColAcc, tmem + 128 * buf + 64, xd, n > 0);
          if (KEYS && fine) {
            add(tmem + kColAcc + D, tmem + 128 * buf + 16, yd, true);
            add(tmem + kColAcc, tmem + 128 * buf + 64 + 16, xd, true);
          }
          tc_commit(s32(&sm.added[buf]));
          tc_commit(s32(&sm.ring_empty[s]));
          if (n == it.chunks - 1) tc_commit(s32(&sm.acc_full));
        }
        __syncwarp();
        if (++s == (uint32_t)S::kSlots) s = 0;
        if (++buf == (uint32_t)kGroups) { buf = 0; buf_phase ^= 1; }
      }
    }
    if (*abort) {
      if (elect_one()) mma_drain(s32(&sm.drain[1]));
      __syncwarp();
    }
  } else if (warp > P::kWMma + 1) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kOtherRegs));
  } else {
    // ------------------------------------------------------------- row threads
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(P::kRowRegs));
    const int grp = warp >> 2, row = tid & 127;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tb = tmem + lane_off + 128 * grp;  // a group's chunks are all in its own buffer
    const uint64_t scale2 = pack2(g.scale_log2, g.scale_log2);
    uint32_t cc = 0, items = 0;
    bool ok = true;
    for (int index = first_item; index < total && ok; index += gridDim.x) {
      it.make(g, a, index);
      const int r = it.row0 + row;
      float nl = 0.f, nd = 0.f;
      if (!KEYS && it.chunks > 0 && row < it.rows) {
        const long long at = ((long long)it.b * g.H + it.head) * a.pad + r;
        nl = __ldg(a.neg_lse2 + at);
        nd = __ldg(a.neg_d + at);
      }
      const uint64_t nl2 = pack2(nl, nl), nd2 = pack2(nd, nd);
      const int first = (grp + kGroups - (int)(cc % kGroups)) % kGroups;
      for (int n = first, j = KEYS ? first % max(it.per, 1) : first; n < it.chunks; n += kGroups) {
        const uint32_t c = cc + n, s = c % S::kSlots;
        int start, cols;
        it.chunk(j, start, cols);
        j += kGroups;
        if (KEYS)
          while (j >= it.per) j -= it.per;
        // columns that the row sees: [from, upto), and the first `sink`; and whether all rows see all of them
        int from, upto, sink = 0;
        bool whole;
        if constexpr (KEYS) {
          from = r - it.off - start;
          upto = r < g.sinks ? cols : min(cols, r + g.window - it.off - start);
          whole = cols == kChunkRows && it.off + start >= it.row0 + kRows - 1 && it.off + start + kChunkRows <= it.row0 + g.window;
        } else {
          const int p = it.off + r;
          from = p - g.window + 1 - start;
          upto = min(cols, p - start + 1);
          sink = g.sinks - start;
          whole = cols == kChunkRows && start + kChunkRows <= it.off + it.row0 + 1 &&
                  (start + kChunkRows <= g.sinks || start > it.off + it.row0 + kRows - 1 - g.window);
        }
        ok = warp_wait_here(s32(&sm.sd_full[grp]), (c / kGroups) & 1, abort, status);
        if (KEYS && ok) ok = warp_wait_here(s32(&sm.ring_full[s]), (c / S::kSlots) & 1, abort, status);  // (landed: for the copies' visibility)
        if (!ok) break;
        tc_fence_after();
        // 32 columns at a time: P and dS, stored in the places of S and dP that have been read
        auto part = [&](int half, auto masked, auto fine) {
          uint32_t sv[32], dv[32], pk[16], dk[16];
          [[maybe_unused]] uint32_t pl[16], dl[16];
          tmem_ld32(tb + 32 * half, sv);
          tmem_ld32(tb + 64 + 32 * half, dv);
          tmem_wait_ld();
          const uint32_t see = low_bits(upto - 32 * half) & (~low_bits(from - 32 * half) | low_bits(sink - 32 * half));
          [[maybe_unused]] const float* st = &sm.stat[s][0][32 * half];
#pragma unroll
          for (int x = 0; x < 32; x += 4) {
            uint64_t l01 = nl2, l23 = nl2, d01 = nd2, d23 = nd2;
            if constexpr (KEYS) {
              const float4 l4 = *reinterpret_cast<const float4*>(st + x), d4 = *reinterpret_cast<const float4*>(st + kChunkRows + x);
              l01 = pack2(l4.x, l4.y); l23 = pack2(l4.z, l4.w);
              d01 = pack2(d4.x, d4.y); d23 = pack2(d4.z, d4.w);
            }
            float y0, y1, y2, y3;
            unpack2(fma2(pack2(__uint_as_float(sv[x]), __uint_as_float(sv[x + 1])), scale2, l01), y0, y1);
            unpack2(fma2(pack2(__uint_as_float(sv[x + 2]), __uint_as_float(sv[x + 3])), scale2, l23), y2, y3);
            float p0 = ex2(y0), p1 = ex2(y1), p2 = ex2(y2), p3 = ex2(y3);
            float e0, e1, e2, e3;
            unpack2(mul2(pack2(p0, p1), add2(pack2(__uint_as_float(dv[x]), __uint_as_float(dv[x + 1])), d01)), e0, e1);
            unpack2(mul2(pack2(p2, p3), add2(pack2(__uint_as_float(dv[x + 2]), __uint_as_float(dv[x + 3])), d23)), e2, e3);
            if (decltype(masked)::value) {
              const bool v0 = (see >> x) & 1u, v1 = (see >> (x + 1)) & 1u, v2 = (see >> (x + 2)) & 1u, v3 = (see >> (x + 3)) & 1u;
              p0 = v0 ? p0 : 0.f; p1 = v1 ? p1 : 0.f; p2 = v2 ? p2 : 0.f; p3 = v3 ? p3 : 0.f;
              e0 = v0 ? e0 : 0.f; e1 = v1 ? e1 : 0.f; e2 = v2 ? e2 : 0.f; e3 = v3 ? e3 : 0.f;
            }
            pk[x >> 1] = pack2<F16>(p0, p1);
            pk[(x >> 1) + 1] = pack2<F16>(p2, p3);
            dk[x >> 1] = pack2<F16>(e0, e1);
            dk[(x >> 1) + 1] = pack2<F16>(e2, e3);
            if constexpr (decltype(fine)::value) {
              pl[x >> 1] = rest<F16>(p0, p1, pk[x >> 1]);
              pl[(x >> 1) + 1] = rest<F16>(p2, p3, pk[(x >> 1) + 1]);
              dl[x >> 1] = rest<F16>(e0, e1, dk[x >> 1]);
              dl[(x >> 1) + 1] = rest<F16>(e2, e3, dk[(x >> 1) + 1]);
            }
          }
          if constexpr (KEYS) tmem_st16(tb + 32 * half, pk);
          tmem_st16(tb + 64 + 32 * half, dk);
          if constexpr (decltype(fine)::value) {
            tmem_st16(tb + 32 * half + 16, pl);
            tmem_st16(tb + 64 + 32 * half + 16, dl);
          }
        };
        if (KEYS && it.holds_sinks(g)) {
          part(0, std::true_type{}, std::integral_constant<bool, KEYS>{});
          part(1, std::true_type{}, std::integral_constant<bool, KEYS>{});
        } else if (whole) {
          part(0, std::false_type{}, std::false_type{});
          part(1, std::false_type{}, std::false_type{});
        } else {
          part(0, std::true_type{}, std::false_type{});
          part(1, std::true_type{}, std::false_type{});
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(s32(&sm.p_full[grp]));
      }
      if (!ok) break;
      cc += it.chunks;
      // results: two groups share dq's columns; or group 0 writes dv, group 1 dk
      if (grp >= 2) continue;
      if (it.chunks > 0) {
        ok = warp_wait_here(s32(&sm.acc_full), items & 1, abort, status);
        if (!ok) break;
        ++items;
        tc_fence_after();
      }
      constexpr int kCols = KEYS ? D : D / 2;
      const uint32_t ta = tmem + lane_off + kColAcc + (KEYS ? (grp ? 0 : D) : grp * (D / 2));
      const View& out = KEYS && grp == 0 ? a.dy0 : a.dx0;
      const float f = KEYS && grp == 0 ? 1.f : g.scale;
      const bool sink_row = KEYS && r < g.sinks && a.pieces > 0 && it.row0 == 0;
      char* dst = out.data + it.b * out.sb + (KEYS ? it.hk : it.head) * out.sh + (long long)r * out.sn + (KEYS ? 0 : grp * D);
      float* sums = a.partial + ((((long long)it.b * g.Hkv + it.hk) * (a.pieces + 1) + it.piece) * 2 + (grp == 0)) * g.sinks * D + (long long)r * D;
#pragma unroll 1
      for (int part = 0; part < kCols / 32; ++part) {
        uint32_t v[32];
        if (it.chunks > 0) {
          tmem_ld32(ta + 32 * part, v);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int x = 0; x < 32; ++x) v[x] = 0u;
        }
        if (row < it.rows && sink_row) {
#pragma unroll
          for (int x = 0; x < 32; x += 4)
            *reinterpret_cast<float4*>(sums + 32 * part + x) = make_float4(__uint_as_float(v[x]) * f, __uint_as_float(v[x + 1]) * f,
                                                                           __uint_as_float(v[x + 2]) * f, __uint_as_float(v[x + 3]) * f);
        } else if (row < it.rows && it.piece == 0) {
#pragma unroll
          for (int x = 0; x < 32; x += 8) {
            uint32_t w[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) w[y] = pack2<F16>(__uint_as_float(v[x + 2 * y]) * f, __uint_as_float(v[x + 2 * y + 1]) * f);
            *reinterpret_cast<uint4*>(dst + 64 * part + 2 * x) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      if (it.chunks > 0) {
        tc_fence_before();
        mbar_arrive(s32(&sm.acc_free));
      }
    }
  }
  cta_tmem_free(warp == P::kWMma, tmem, kTmemCols);
}

// -lse in base 2 and -D = -<dO, O> of every row, eight lanes a row and kRowsAhead rows a lane.  Rows that do not exist, and rows that
// see nothing (whose weights are masked whatever stands here), get zeros.  Clears the status block.
namespace {
constexpr int kRowsAhead = 4;
template <int D, bool F16>
__global__ void __launch_bounds__(256) window_rows_kernel(const WinGeo g, const View o, const View d_o, const float* __restrict__ lse,
                                                          float* __restrict__ neg_lse2, float* __restrict__ neg_d, int pad, unsigned blocks,
                                                          int* status) {
  const unsigned cta = blockIdx.x + (unsigned)await_stream();
  const int unit = (int)(cta / blocks), b = unit / g.H, h = unit - b * g.H;
  const int first = (int)(cta - unit * blocks) * (32 * kRowsAhead) + (threadIdx.x >> 3), part = threadIdx.x & 7;
  if (blockIdx.x == 0 && threadIdx.x < kStatusBytes / 4) status[threadIdx.x] = 0;
  const int ql = span_of(g, b).ql;
  const char *x = o.data + b * o.sb + h * o.sh + 16 * part, *y = d_o.data + b * d_o.sb + h * d_o.sh + 16 * part;
  uint4 u[kRowsAhead][D / 64], w[kRowsAhead][D / 64];
  float l[kRowsAhead];
#pragma unroll
  for (int r = 0; r < kRowsAhead; ++r) {
    const int i = first + 32 * r;
    l[r] = i < ql ? __ldg(lse + (long long)unit * g.Nq + i) : 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      u[r][c] = w[r][c] = make_uint4(0u, 0u, 0u, 0u);
      if (i < ql) {
        u[r][c] = __ldg(reinterpret_cast<const uint4*>(x + (long long)i * o.sn + 128 * c));
        w[r][c] = __ldg(reinterpret_cast<const uint4*>(y + (long long)i * d_o.sn + 128 * c));
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kRowsAhead; ++r) {
    float dot = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const uint32_t uw[4] = {u[r][c].x, u[r][c].y, u[r][c].z, u[r][c].w}, ww[4] = {w[r][c].x, w[r][c].y, w[r][c].z, w[r][c].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float u0, u1, w0, w1;
        unpack16x2(uw[k], F16, u0, u1);
        unpack16x2(ww[k], F16, w0, w1);
        dot = fmaf(u0, w0, fmaf(u1, w1, dot));
      }
    }
#pragma unroll
    for (int k = 4; k; k >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, k);
    const int i = first + 32 * r;
    if (part == 0 && i < pad) {
      neg_lse2[(long long)unit * pad + i] = l[r] == -INFINITY ? 0.f : -l[r] * 1.4426950408889634f;
      neg_d[(long long)unit * pad + i] = -dot;
    }
  }
}

// The sinks' gradients: the window's part and the pieces', in order.
template <int D, bool F16>
__global__ void __launch_bounds__(256) window_sinks_kernel(const WinGeo g, const __grid_constant__ BwdArgs a) {
  const int unit = (int)blockIdx.x + await_stream(), b = unit / g.Hkv, hk = unit - b * g.Hkv;
  const Span s = span_of(g, b);
  const int left = s.ql - first_tile_end(g, s), pieces = left > 0 ? (left + a.piece_rows - 1) / a.piece_rows : 0;
  const int n = min(g.sinks, s.kl) * D, step = g.sinks * D;
  const float* p = a.partial + (long long)unit * (a.pieces + 1) * 2 * step;
  for (int e = 2 * (blockIdx.y * 256 + threadIdx.x); e < 2 * n; e += 512 * gridDim.y) {
    const int which = e >= n, x = e - which * n;  // 0: dk, 1: dv; two channels
    float2 v = make_float2(0.f, 0.f);
    for (int k = 0; k <= pieces; ++k) {
      const float2 w = *reinterpret_cast<const float2*>(p + (long long)(2 * k + which) * step + x);
      v.x += w.x;
      v.y += w.y;
    }
    const View& out = which ? a.dy0 : a.dx0;
    *reinterpret_cast<uint32_t*>(out.data + b * out.sb + hk * out.sh + (long long)(x / D) * out.sn + 2 * (x % D)) = pack2<F16>(v.x, v.y);
  }
}

template <int D, bool F16, bool KEYS>
int launch_pass(const HostCtx& c, const WinGeo& g, const View& x0, const View& y0, const View& x, const View& y, const BwdArgs& a) {
  CUtensorMap mx0, my0, mx, my;
  const int h0 = KEYS ? g.Hkv : g.H, h1 = KEYS ? g.H : g.Hkv, n0 = KEYS ? g.Nk : g.Nq, n1 = KEYS ? g.Nq : g.Nk;
  if (!make_map_view(&mx0, x0, D, n0, h0, g.B, kRows) || !make_map_view(&my0, y0, D, n0, h0, g.B, kRows) ||
      !make_map_view(&mx, x, D, n1, h1, g.B, kChunkRows) || !make_map_view(&my, y, D, n1, h1, g.B, kChunkRows))
    return MOSAIC_E_CUDA;
  const size_t smem = sizeof(Smem<D>) + 1024;
  static unsigned long long configured = 0;
  int sms = 0;
  const void* func = reinterpret_cast<const void*>(window_bwd_kernel<D, F16, KEYS>);
  if (const int rc = launch_setup_regs(func, Plan<D, KEYS>::kLaunchRegs, smem, &configured, &sms)) return rc;
  const long long total = (long long)g.B * h0 * (a.tiles + a.pieces);
  if (total > 0x7ffffff0ll) return MOSAIC_E_UNSUPPORTED;
  return launch_kernel(window_bwd_kernel<D, F16, KEYS>, dim3((unsigned)(total < sms ? total : sms)), Plan<D, KEYS>::kThreads, smem, c.stream, true, 0, g,
                       mx0, my0, mx, my, fold_of(x0), fold_of(y0), fold_of(x), fold_of(y), a, c.status, (int)total);
}

template <int D, bool F16>
int launch(const HostCtx& c, const WinGeo& g, const WinBwd& t, const WinBwdWs& w, char* ws) {
  const unsigned blocks = (unsigned)((w.pad + 32 * kRowsAhead - 1) / (32 * kRowsAhead));  // of a unit's rows
  if ((long long)blocks * g.B * g.H > 0x7fffffffll) return MOSAIC_E_UNSUPPORTED;
  float *nl = (float*)(ws + w.neg_lse2), *nd = (float*)(ws + w.neg_d);
  int rc = launch_kernel(window_rows_kernel<D, F16>, dim3(blocks * (unsigned)(g.B * g.H)), 256, 0, c.stream, true, 0, g, t.o, t.d_o, t.lse, nl, nd,
                         w.pad, blocks, c.status);
  if (rc) return rc;
  BwdArgs a = {t.dk, t.dv, nl, nd, (float*)(ws + w.partial), w.pad, (g.Nk + kRows - 1) / kRows, w.pieces, w.piece_rows};
  if ((rc = launch_pass<D, F16, true>(c, g, t.k, t.v, t.q, t.d_o, a))) return rc;
  if (w.pieces > 0) {
    const int split = (2 * g.sinks * D + 511) / 512;
    rc = launch_kernel(window_sinks_kernel<D, F16>, dim3((unsigned)(g.B * g.Hkv), (unsigned)split), 256, 0, c.stream, true, 0, g, a);
    if (rc) return rc;
  }
  a.dx0 = t.dq;
  a.tiles = (g.Nq + kRows - 1) / kRows;
  a.pieces = 0;
  return launch_pass<D, F16, false>(c, g, t.q, t.d_o, t.k, t.v, a);
}
}  // namespace

WinBwdWs window_bwd_layout(const WinGeo& g) {
  WinBwdWs w;
  w.pad = (g.Nq + kRows - 1) / kRows * kRows;
  // A piece of the sinks' further rows is as long as a tile's own list of a head.  Rows beyond tile 0's list have positions from
  // kRows - 1 + window on; how many there are is only known on the device, this is the most.
  w.piece_rows = (int)(((long long)g.window + kRows + kChunkRows - 1) / kChunkRows * kChunkRows);
  const int behind = g.Nk - (kRows - 1) - g.window, beyond = behind < g.Nq ? behind : g.Nq;
  w.pieces = g.sinks > 0 && beyond > 0 ? (beyond + w.piece_rows - 1) / w.piece_rows : 0;
  size_t at = kStatusBytes;
  w.neg_lse2 = at; at = align256(at + sizeof(float) * (size_t)g.B * g.H * w.pad);
  w.neg_d = at; at = align256(at + sizeof(float) * (size_t)g.B * g.H * w.pad);
  w.partial = at; at = align256(at + (w.pieces > 0 ? sizeof(float) * (size_t)g.B * g.Hkv * (w.pieces + 1) * 2 * g.sinks * g.d : 0));
  w.total = at;
  return w;
}

int launch_window_bwd(const HostCtx& c, const WinGeo& g, bool f16, const WinBwd& t, void* ws) {
  const WinBwdWs w = window_bwd_layout(g);
  if (g.d == 64) return f16 ? launch<64, true>(c, g, t, w, (char*)ws) : launch<64, false>(c, g, t, w, (char*)ws);
  return f16 ? launch<128, true>(c, g, t, w, (char*)ws) : launch<128, false>(c, g, t, w, (char*)ws);
}

}  // namespace mosaic
