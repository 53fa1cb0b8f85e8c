// Attention of one or a few new tokens per sequence over a paged cache, and the join of its parts.
//
//   o_i = sum_j exp(scale q_i . k_j - m_i) v_j / l_i  over the keys that row i sees: j <= p_i, and p_i - j < window or j < sinks
// HBM-bound: the visible keys and values of a key/value head are read once for each block of its rows (new tokens x query heads of the
// group; up to 16 at D = 128 and 32 at 64 are one block), by further blocks from the L2.  The keys of a member are cut into chunks of 512; a chunk of a head is an item.  Persistent CTAs, one an SM,
// take equal shares of the list of all items, which each works out from the lengths.
//
// One warp finds the items, and for each leaves a note of what the others need to know of it, with the numbers of its pages, and copies its
// queries.  Two ask for the items' steps of 64 keys by TMA, page by page, into a ring that all warps share, one for keys and one for
// values; they run ahead of the others, so that the memory never waits for a chunk's end.  The others take the chunk's steps in turn, a
// step each: products of 16 x 8 x 16 are enough,
//   S^T = K Q^T (16 keys x 8 rows), O^T += V^T P^T (16 channels x 8 rows), P^T turned from accumulator to operand by a transpose,
// and the step's 64 keys give every lane four of them that do not wait for one another.  Weights round to 16 bits once, as operands;
// everything else is fp32.  The warps' maxima, sums and accumulators are joined through shared memory at the chunk's end, and leave as a
// part; a second kernel joins a row's parts in their order.  Members that can have one part only get their results at once, joined with
// the prefix' parts if there is a prefix.
//
// Measured (us on the device, 4 key/value heads of 128 unless given): 64 members of up to 8192 tokens, 16 heads, pages of 64, 106.8, and 8
// of 65536, 32 heads, 188; in the steady state a chunk (262 KB) takes an SM 10100 cycles, 7.4 TB/s in all.  One member of 16384, 12.6:
// 5000 cycles until the first copies are asked for, 600 a step, 2000 for the last step and the join, 4000 the second kernel.  5 new tokens of
// 32 members, 12 heads on 3 of 64, window 2048: 27.
// Tried on the last of these, with what it took then and what it takes without: rings and steps of 16 keys for every warp 63 (44), all
// warps finding the items 46 (38), copies by one lane 35 (31), one more warp for the join of a chunk's steps 55 (31), conditions of the
// masks and of the join as branches 33 (29).
#include <type_traits>

#include "mma16.cuh"
#include "paged.cuh"

namespace mosaic {

namespace {

constexpr int kStep = 64, kSteps = kChunkKeys / kStep;
// Barriers on which steps land, in turn.  A warp looks at its own steps only, and a wait on a phase's parity is exact only if the
// barrier's phase before has completed: that is sure if it belongs to an earlier chunk, whose steps have all been taken.
constexpr int kBars = 16;
static_assert(kChunkKeys / kMinPage == 32, "a lane has a box");
static_assert(kBars >= kSteps, "a step's barrier has been used by an earlier one of the chunk");
constexpr int kMaxSmem = 232448;

constexpr int kJobs = 4;  // items that the first warp may be ahead

// What the others need to know of an item
struct alignas(16) Note {
  int b, head0, rb, part;  // member, first query head of the group, block of rows, place among all parts
  int kl, ql, p0, from;    // as in Parts
  int sinks, key0;         // first position of the chunk
  unsigned steps;          // of the chunk, that any row sees something of
  int more;                // 0: no item, and none will come
};
struct Job {
  Note note;
  int page[kChunkKeys / kMinPage];  // of the chunk's boxes; g.pages, behind the last: none, or no row sees anything of it
};

// NT: tiles of 8 rows that a CTA takes
template <int D, int NT>
struct Smem {
  static constexpr int kWarps = 8;  // that take steps
  static constexpr int kThreads = 32 * (kWarps + 3);
  static constexpr int kHalf = kStep * D * 2, kStepBytes = 2 * kHalf;  // a step's keys, then its values
  static constexpr int kPitch = D + 4;  // of a row of part_o: lanes that store side by side meet different banks
  static constexpr int kRowBytes = D * 2;
  static constexpr int kOther = 4 * kWarps * 8 * NT * (kPitch + 2) + kJobs * (8 * NT * kRowBytes + (int)sizeof(Job)) + 1024;
  static constexpr int kRoom = (kMaxSmem - 1024 - kOther) / kStepBytes, kStages = kRoom < 12 ? kRoom : 12;
  unsigned char ring[kStages][kStepBytes];
  unsigned char q[kJobs][8 * NT * kRowBytes];  // 16-byte pieces of a row swizzled by its number
  float part_o[kWarps][8 * NT][kPitch], part_m[kWarps][8 * NT], part_l[kWarps][8 * NT];
  Job job[kJobs];
  unsigned long long full[kBars], empty[kStages], note_full[kJobs], job_full[kJobs], job_empty[kJobs], parts_full, parts_read;
  unsigned hole[kStages];  // the step's boxes that have no page
  long long scan[kWarps + 3];
  int4 start;              // the member that this CTA's share begins in, the weight before it, its lengths
  int abort;
};

struct DecArgs {
  View q, o;
  float* lse;
  PartsOut parts;
  int blocks;     // of rows
  int box_shift;  // log2 of the slots that a copy brings: a page, at most a step
  int turn;       // weight of an item beside its steps; 0: all items weigh the same
  bool direct, first;
  float inv_g;    // 1 / G
  int* status;
};

// A place in the list of all items: members, their heads, their parts, blocks of rows.  An item weighs `turn` for what comes with every one
// and `mul` times its steps; `pos` is the weight of all items before.
__device__ __forceinline__ Parts parts_of(const PagedGeo& g, const DecArgs& a, const Span& s) {
  Parts p = parts_of(g, s);
  if (a.direct) p.n = p.ql > 0 ? 1 : 0;  // (a member without keys has results too)
  return p;
}
struct Walk {
  Parts p;
  int b, hk, o, rb, pos, mul, turn;
  int held, kl, ql;  // lengths of the 32 members from `held` on, in the lanes, as they stand in memory (nothing waits for them here)
  __device__ __forceinline__ void hold(const PagedGeo& g) {
    held = b;
    const int m = min(b + (int)(threadIdx.x & 31), g.B - 1);
    kl = __ldg(g.k_len + m);
    ql = g.q_len ? __ldg(g.q_len + m) : g.T;
  }
  __device__ __forceinline__ void member(const PagedGeo& g, const DecArgs& a) {
    if (b - held >= 32) hold(g);
    p = parts_of(g, a, clamped(g, __shfl_sync(0xffffffffu, kl, b - held), __shfl_sync(0xffffffffu, ql, b - held)));
  }
  __device__ __forceinline__ int weight(int part) const {
    if (p.front && part == 0) return mul * ((p.sinks + kStep - 1) / kStep) + turn;
    const int s = chunk_of(p, part) * kSteps;
    return mul * (min(s + kSteps - 1, (p.kl - 1) >> 6) - max(s, p.from >> 6) + 1) + turn;
  }
  // of the parts before `part`: only the first two and the last may be short
  __device__ __forceinline__ int weight_before(int part) const {
    return part == 0 ? 0 : part == 1 ? weight(0) : weight(0) + weight(1) + (part - 2) * (mul * kSteps + turn);
  }
  __device__ __forceinline__ int weight_of_head(const DecArgs& a) const { return p.n ? a.blocks * (weight_before(p.n - 1) + weight(p.n - 1)) : 0; }
  // To the first item of the member (of weight `base` before it) that does not begin before weight `to`, or behind the member
  __device__ __forceinline__ void seek(const PagedGeo& g, const DecArgs& a, int base, int to) {
    const int head = weight_of_head(a), at = max(to - base, 0);
    hk = at / head;
    const int y = at - hk * head;
    o = 0;
    if (p.n > 2 && y >= a.blocks * weight_before(2)) o = min(p.n - 1, 2 + (y - a.blocks * weight_before(2)) / (a.blocks * (mul * kSteps + turn)));
    else if (p.n > 1 && y >= a.blocks * weight_before(1)) o = 1;
    const int rest = y - a.blocks * weight_before(o), each = weight(o);
    rb = (rest + each - 1) / each;
    pos = base + hk * head + a.blocks * weight_before(o) + rb * each;
    if (rb == a.blocks) {
      rb = a.blocks - 1;
      pos -= each;
      next(g, a);
    }
  }
  __device__ __forceinline__ void next(const PagedGeo& g, const DecArgs& a) {
    pos += weight(o);
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
  __device__ __forceinline__ int key0() const { return chunk_of(p, o) * kChunkKeys; }
  // any row sees some of the n keys from j on
  __device__ __forceinline__ bool seen(int j, int n) const { return j < p.kl && (j + n > p.from || j < p.sinks); }
  // the chunk's steps that are, by the whole warp
  __device__ __forceinline__ unsigned steps(int lane) const {
    return __ballot_sync(0xffffffffu, lane < kSteps && seen(key0() + lane * kStep, kStep));
  }
};
static_assert(kStep == 64 && kBoxShift == 6, "weights count steps by shifts");

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// Sum of v over the threads before this one, and over all
template <int WARPS>
__device__ __forceinline__ long long block_scan(long long v, long long* scan, long long& total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long x = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) scan[warp] = x;
  __syncthreads();
  long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    before += w < warp ? scan[w] : 0;
    total += scan[w];
  }
  return before + x - v;
}

// A row's result is its sums over the sum of weights (a sum that is not a number stays one)
__device__ __forceinline__ float inverse_of(float sum) { return sum <= 0.f ? 0.f : 1.f / sum; }
__device__ __forceinline__ float lse_of(float m, float sum) { return sum <= 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f; }

template <int D, bool F16, int NT>
__global__ void __launch_bounds__(Smem<D, NT>::kThreads, 1)
    paged_parts_kernel(const PagedGeo g, const __grid_constant__ DecArgs a, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v) {
  using S = Smem<D, NT>;
  constexpr int kRowsCta = 8 * NT, kStages = S::kStages, kWarps = S::kWarps;
  extern __shared__ unsigned char smem_raw[];
  S& sm = *reinterpret_cast<S*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gq = lane >> 2, tq = lane & 3;
  if (tid == 0) {
    for (int s = 0; s < kBars; ++s) mbar_init(s32(&sm.full[s]), 2);  // keys and values
    for (int s = 0; s < kStages; ++s) mbar_init(s32(&sm.empty[s]), 1);
    for (int s = 0; s < kJobs; ++s) {
      mbar_init(s32(&sm.note_full[s]), 1);
      mbar_init(s32(&sm.job_full[s]), 33);  // the note, and every lane's copies
      mbar_init(s32(&sm.job_empty[s]), kWarps + 2);
    }
    mbar_init(s32(&sm.parts_full), kWarps);
    mbar_init(s32(&sm.parts_read), kWarps);
    sm.abort = 0;
    cta_publish_barriers();
  }
  __syncthreads();
  // (behind a prefix the kernel ahead is the prefix', whose results only the join reads)
  const int zero = a.first ? await_stream() : pass_stream();
  // A code is written no earlier than a wait's bound of seconds after its CTA began; the first CTA has cleared the word by then.
  if (a.first && blockIdx.x == 0 && tid == 0) a.status[zero] = 0;
  volatile int* abort = &sm.abort;

  const int rows = g.G * g.T;

  // ---- this CTA's share of the list: the items that begin in its share of the weight.  Where there are no more items than CTAs, each has
  // one at most.
  int begin, end, mul, turn;
  {
    Span s = {};
    long long mine = 0, before = 0, total = 0;  // items in the upper half, their steps in the lower one
    auto weigh = [&](int b) {
      mine = 0;
      if (b < g.B) {
        Walk w;
        s = span_of(g, b);
        w.p = parts_of(g, a, s);
        w.mul = 1;
        w.turn = 0;
        mine = (long long)w.p.n * a.blocks * g.Hkv << 32 | (unsigned)(w.weight_of_head(a) * g.Hkv);
      }
    };
#pragma unroll 1
    for (int b0 = 0; b0 < g.B; b0 += S::kThreads) {
      long long all;
      weigh(b0 + tid + zero);
      if (b0) __syncthreads();
      before = block_scan<kWarps + 3>(mine, sm.scan, all);
      total += all;
    }
    mul = a.turn && total >> 32 > gridDim.x;
    turn = mul ? a.turn : 1;
    auto weight = [&](long long x) { return mul * (int)(unsigned)x + turn * (int)(x >> 32); };
    begin = (int)((long long)weight(total) * blockIdx.x / gridDim.x);
    end = (int)((long long)weight(total) * (blockIdx.x + 1) / gridDim.x);
    int base = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < g.B; b0 += S::kThreads) {
      long long all = 0;
      if (g.B > S::kThreads) {
        weigh(b0 + tid + zero);
        __syncthreads();
        before = block_scan<kWarps + 3>(mine, sm.scan, all);
      }
      const int at = begin - base - weight(before);
      if (at >= 0 && at < weight(mine)) sm.start = make_int4(b0 + tid, base + weight(before), s.kl, s.ql);
      base += weight(all);
    }
    __syncthreads();
  }

  if (warp == kWarps) {
    // ------------------------------------------------------------- items
    const int box = 1 << a.box_shift, boxes = kChunkKeys >> a.box_shift;  // a lane has one of the chunk's boxes
    Walk w;
    w.pos = end;
    w.mul = mul;
    w.turn = turn;
    if (begin < end) {
      const int4 at = sm.start;
      w.b = at.x;
      w.p = parts_of(g, a, Span{at.w, at.z, at.z - at.w});
      w.hold(g);
      w.seek(g, a, at.y, begin);
    }
#ifdef MOSAIC_TEST_WITHHOLD_FIRST_LIST
    bool ok = false;  // test build only: nothing is ever handed out or loaded, so that every wait for it runs out
#else
    bool ok = true;
#endif
    // the page of this lane's box
    auto look_up = [&]() {
      const int key = w.key0() + (lane << a.box_shift);
      return lane < boxes && w.seen(key, box) ? __ldg(g.table + w.b * g.table_stride + (key >> g.shift)) : -1;
    };
    uint32_t slot = 0, round = 0;
    bool more = w.pos < end;
    int id = more ? look_up() : 0;
#pragma unroll 1
    while (ok) {
      ok = warp_wait(s32(&sm.job_empty[slot]), round ^ 1, abort, a.status);
      if (!ok) break;
      const uint32_t job_bar = s32(&sm.job_full[slot]);
      const unsigned steps = more ? w.steps(lane) : 0u;
      sm.job[slot].page[lane] = (unsigned)id < (unsigned)g.pages ? id : g.pages;
      if (lane == 0) {
        Note n;
        n.b = w.b; n.head0 = w.hk * g.G; n.rb = w.rb; n.part = a.parts.shared + w.o;
        n.kl = w.p.kl; n.ql = w.p.ql; n.p0 = w.p.p0; n.from = w.p.from;
        n.sinks = w.p.sinks; n.key0 = w.key0(); n.steps = steps; n.more = more;
        sm.job[slot].note = n;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(s32(&sm.note_full[slot]));
      if (more) {  // the queries: row by row, whatever their strides
        const uint32_t dst = s32(sm.q[slot]);
        const char* src = a.q.data + w.b * a.q.sb + w.hk * g.G * a.q.sh;
#pragma unroll
        for (int e0 = 0; e0 < kRowsCta * D / 8; e0 += 32) {
          const int e = e0 + lane, row = e / (D / 8), c = e % (D / 8), r = min(w.rb * kRowsCta + row, rows - 1);
          const int i = g.T == 1 ? 0 : quick_div(r, g.G, a.inv_g);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + row * S::kRowBytes + ((c ^ (row & 7)) << 4)),
                       "l"(src + (r - i * g.G) * a.q.sh + i * a.q.sn + 16 * c)
                       : "memory");
        }
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(job_bar) : "memory");
      if (lane == 0) mbar_arrive(job_bar);
      if (!more) break;
      if (++slot == kJobs) { slot = 0; round ^= 1; }
      w.next(g, a);
      more = w.pos < end;
      if (more) id = look_up();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");  // copies must have landed before the CTA's memory is released
    if (!a.first) settle_stream();
    return;
  }
  if (warp > kWarps) {
    // ------------------------------------------------------------- copies: of keys the first warp, of values the second
    const bool values = warp == kWarps + 2;
    const CUtensorMap* map = values ? &map_v : &map_k;
    const int boxes = kStep >> a.box_shift, in_page = (1 << g.shift) - 1;
    const uint32_t box_bytes = (uint32_t)(D * 2) << a.box_shift;
    uint32_t stage = 0, phase = 0, issued = 0, slot = 0, round = 0;
    bool ok = true;
#pragma unroll 1
    while (ok) {
      ok = warp_wait(s32(&sm.note_full[slot]), round, abort, a.status);
      if (!ok) break;
      const Note& job = sm.job[slot].note;
      if (!job.more) break;
      const int page = sm.job[slot].page[lane], hk = quick_div(job.head0, g.G, a.inv_g), at = (job.key0 + (lane << a.box_shift)) & in_page;
      const unsigned holes = __ballot_sync(0xffffffffu, page >= g.pages);
      for (unsigned todo = job.steps; todo; todo &= todo - 1) {
        const int s = __ffs(todo) - 1, first = s * boxes;
        ok = warp_wait(s32(&sm.empty[stage]), phase ^ 1, abort, a.status);
        if (!ok) break;
        const uint32_t bar = s32(&sm.full[issued % kBars]), dst = s32(sm.ring[stage]) + (values ? S::kHalf : 0) + (lane - first) * box_bytes;
        if (lane == 0) {
          if (!values) sm.hole[stage] = (holes >> first) & low_bits(boxes);
          mbar_expect_tx(bar, S::kHalf);
        }
        __syncwarp();
        if (lane >= first && lane < first + boxes) load_slots(dst, map, bar, at, 0, hk, page);  // (rows behind the last page arrive as zeros)
        ++issued;
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(s32(&sm.job_empty[slot]));
      if (++slot == kJobs) { slot = 0; round ^= 1; }
    }
    // copies must have landed before the CTA's memory is released (their readers have waited for them, unless a wait ran out)
    if (*abort && lane == 0)
      for (uint32_t n = issued > kStages ? issued - kStages : 0; n < issued; ++n) mbar_drain(s32(&sm.full[n % kBars]), (n / kBars) & 1);
    if (!a.first) settle_stream();
    return;
  }

  // ------------------------------------------------------------- steps
  uint32_t taken = 0, slot = 0, round = 0, joins = 0;  // steps of the items so far, all warps'; items
  const int box = 1 << a.box_shift;
  const uint32_t ka = (uint32_t)((lane & 15) * 128), kx = (uint32_t)(lane & 7), kh = (uint32_t)(lane >> 4);           // keys as they lie
  const uint32_t va = (uint32_t)(((lane & 7) + 8 * (lane >> 4)) * 128), vh = (uint32_t)((lane >> 3) & 1);             // values transposed
  const uint32_t qa = (uint32_t)((lane & 7) * S::kRowBytes), qh = (uint32_t)(lane >> 3);                              // four pieces of 8 rows
#pragma unroll 1
  for (;; ++joins) {
    if (!warp_wait(s32(&sm.job_full[slot]), round, abort, a.status)) break;
    const Note job = sm.job[slot].note;
    if (!job.more) break;
    const unsigned steps = job.steps;
    float m[NT][2], l[NT][2], acc[NT][D / 16][4];
    if ((steps >> warp) & 1u) {
      const int j0 = job.key0 + warp * kStep;
      const uint32_t at = taken + __popc(steps & low_bits(warp)), stage = at % kStages;
      if (!warp_wait(s32(&sm.full[at % kBars]), (at / kBars) & 1, abort, a.status)) break;
      const uint32_t kt = s32(sm.ring[stage]), vt = kt + S::kHalf, qt = s32(sm.q[slot]);
      const unsigned hole = sm.hole[stage];
      // all rows see all of the step
      const bool whole = !hole && j0 + kStep - 1 <= job.p0 && (!g.window || j0 >= job.kl - g.window || j0 + kStep <= job.sinks);
      // a step's rows lie box by box, a box's 64-channel parts one behind the other
      uint32_t tile[4];  // of 16 keys
#pragma unroll
      for (int k = 0; k < 4; ++k) tile[k] = D == 64 ? 2048u * k : ((16u * k) >> a.box_shift) * ((uint32_t)(D * 2) << a.box_shift) + ((16u * k) & (box - 1)) * 128u;
      const uint32_t part = box * 128u;
      float z[NT][4][4];  // [keys 16 k ..]: (key gq, row 2 tq), (gq, 2 tq + 1), (gq + 8, 2 tq), (gq + 8, 2 tq + 1)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) z[nt][k][0] = z[nt][k][1] = z[nt][k][2] = z[nt][k][3] = 0.f;
#pragma unroll
      for (int c2 = 0; c2 < D / 32; ++c2) {
        uint32_t qf[NT][4];  // 32 channels of 8 rows
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) ldsm4(qf[nt], qt + nt * 8 * S::kRowBytes + qa + (((4 * c2 + qh) ^ kx) << 4));
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int c = 2 * c2 + y;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t f[4];
            ldsm4(f, kt + (c >> 2) * part + tile[k] + ka + (((2 * (c & 3) + kh) ^ kx) << 4));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816<F16>(z[nt][k], f[0], f[1], f[2], f[3], qf[nt][2 * y], qf[nt][2 * y + 1]);
          }
        }
      }
      uint32_t pt[NT][4][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (!whole) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            // the row sees the lane's keys j0 + gq + n for n <= to, and n > to - window or n < sinks
            const int r = job.rb * kRowsCta + 8 * nt + 2 * tq + x, i = g.T == 1 ? 0 : quick_div(r, g.G, a.inv_g);
            const int to = (r < rows && i < job.ql ? job.p0 + i : -1) - j0 - gq, from = g.window ? to - g.window : -1, sinks = job.sinks - j0 - gq;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int n = 16 * k + 8 * y;
                const bool hidden = (n > to) | ((n <= from) & (n >= sinks)) | (bool)((hole >> (16 * k >> a.box_shift)) & 1u);
                z[nt][k][x + 2 * y] = hidden ? -INFINITY : z[nt][k][x + 2 * y];
              }
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float mx = fmaxf(z[nt][0][x], z[nt][0][x + 2]);
#pragma unroll
          for (int k = 1; k < 4; ++k) mx = max3(mx, z[nt][k][x], z[nt][k][x + 2]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16)) * g.scale_log2;  // scale > 0 commutes with max
          m[nt][x] = mx;
          const float ref = mx == -INFINITY ? 0.f : -mx;  // (nothing seen)
          float sum = 0.f;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            z[nt][k][x] = ex2(fmaf(z[nt][k][x], g.scale_log2, ref));
            z[nt][k][x + 2] = ex2(fmaf(z[nt][k][x + 2], g.scale_log2, ref));
            sum += z[nt][k][x] + z[nt][k][x + 2];
          }
          l[nt][x] = sum;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          pt[nt][k][0] = transpose8(pack2<F16>(z[nt][k][0], z[nt][k][1]));
          pt[nt][k][1] = transpose8(pack2<F16>(z[nt][k][2], z[nt][k][3]));
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) acc[nt][c][0] = acc[nt][c][1] = acc[nt][c][2] = acc[nt][c][3] = 0.f;
      }
      auto sums = [&](auto edge) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          // A weight of zero does not silence what is no number: on an edge, values that no row sees become zeros.  A lane has the
          // neighbouring keys 16 k + 2 tq and 8 more.
          uint32_t keep[2] = {};
          if constexpr (decltype(edge)::value) {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int j = j0 + 16 * k + 2 * tq + (y & 1) + 4 * (y & 2);
              keep[y >> 1] |= (j < job.kl) & ((j >= job.from) | (j < job.sinks)) ? 0xffffu << (16 * (y & 1)) : 0u;
            }
          }
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            uint32_t f[4];
            ldsm4t(f, vt + (c >> 2) * part + tile[k] + va + (((2 * (c & 3) + vh) ^ kx) << 4));
            if constexpr (decltype(edge)::value) {
              f[0] &= keep[0]; f[1] &= keep[0];
              f[2] &= keep[1]; f[3] &= keep[1];
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816<F16>(acc[nt][c], f[0], f[1], f[2], f[3], pt[nt][k][0], pt[nt][k][1]);
          }
        }
      };
      if (whole) sums(std::false_type{});
      else sums(std::true_type{});
      __syncwarp();  // the stage has been read
      if (lane == 0) mbar_arrive(s32(&sm.empty[stage]));

      // what the step leaves for the join, once all warps have read the item before's
      if (!warp_wait(s32(&sm.parts_read), (joins & 1) ^ 1, abort, a.status)) break;
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
    }
    taken += __popc(steps);
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(s32(&sm.parts_full));
      mbar_arrive(s32(&sm.job_empty[slot]));
    }
    if (++slot == kJobs) { slot = 0; round ^= 1; }
    if (!warp_wait(s32(&sm.parts_full), joins & 1, abort, a.status)) break;
    // D / 4 lanes have a row; the eight lanes of a group work out the warps' factors, one each
#pragma unroll
    for (int e = tid; e < kRowsCta * D / 4; e += 32 * kWarps) {
      const int h = e / (D / 4), c = 4 * (e - h * (D / 4)), r = job.rb * kRowsCta + h, i = g.T == 1 ? 0 : quick_div(r, g.G, a.inv_g);
      const bool there = (steps >> (lane & 7)) & 1u;
      const float my = there ? sm.part_m[lane & 7][h] : -INFINITY;
      float mx = my;
#pragma unroll
      for (int d = 1; d < 8; d *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      const float factor = my == -INFINITY ? 0.f : ex2(my - mx);
      float sum = there ? sm.part_l[lane & 7][h] * factor : 0.f;
#pragma unroll
      for (int d = 1; d < 8; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int y = 0; y < kWarps; ++y) {  // (without branches, so that the loads overlap; what a warp has not left is not looked at)
        const bool on = (steps >> y) & 1u;
        const float f = __shfl_sync(0xffffffffu, factor, (lane & 24) | y);
        const float4 u = *reinterpret_cast<const float4*>(&sm.part_o[y][h][c]);
        v.x = on ? fmaf(u.x, f, v.x) : v.x;
        v.y = on ? fmaf(u.y, f, v.y) : v.y;
        v.z = on ? fmaf(u.z, f, v.z) : v.z;
        v.w = on ? fmaf(u.w, f, v.w) : v.w;
      }
      const bool live = r < rows && i < job.ql;
      const int head = job.head0 + r - i * g.G;
      const long long row = ((long long)job.b * g.H + head) * g.T + i;
      if (a.direct && a.parts.shared) {
        // the prefix' parts, D / 4 at a time: a lane of the row works out one's factor
        constexpr int L = D / 4, A = 8;
        settle_stream();
        const int mine = lane % L, base = lane - mine;
        const float2* ml = a.parts.ml + row;
        const float* src = a.parts.o + row * D + c;
#pragma unroll 1
        for (int y0 = 0; y0 < a.parts.shared; y0 += L) {
          const int n = min(L, a.parts.shared - y0);
          float4 u[A];
          auto ask = [&](int z0) {  // (behind the last: that again, with a factor of zero)
#pragma unroll
            for (int z = 0; z < A; ++z) {
              u[z] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (live) u[z] = __ldcg(reinterpret_cast<const float4*>(src + (y0 + min(z0 + z, n - 1)) * a.parts.rows * D));
            }
          };
          ask(0);
          float2 part = make_float2(-INFINITY, 0.f);
          if (live && mine < n) part = __ldcg(ml + (y0 + mine) * a.parts.rows);
          float top = fmaxf(mx, part.x);
#pragma unroll
          for (int d = 1; d < L; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          const float own = mx == -INFINITY ? 0.f : ex2(mx - top), f = part.x == -INFINITY ? 0.f : ex2(part.x - top);
          float more = part.y * f;
#pragma unroll
          for (int d = 1; d < L; d *= 2) more += __shfl_xor_sync(0xffffffffu, more, d);
          mx = top;
          sum = fmaf(sum, own, more);
          v.x *= own; v.y *= own; v.z *= own; v.w *= own;
#pragma unroll 1
          for (int z0 = 0; z0 < n; z0 += A) {
            if (z0) ask(z0);
#pragma unroll
            for (int z = 0; z < A; ++z) {
              const float fz = __shfl_sync(0xffffffffu, f, base + z0 + z);
              v.x = fmaf(u[z].x, fz, v.x);
              v.y = fmaf(u[z].y, fz, v.y);
              v.z = fmaf(u[z].z, fz, v.z);
              v.w = fmaf(u[z].w, fz, v.w);
            }
          }
        }
      }
      if (!live) continue;
      if (a.direct) {
        const float inv = inverse_of(sum);
        *reinterpret_cast<uint2*>(a.o.data + job.b * a.o.sb + head * a.o.sh + i * a.o.sn + 2 * c) =
            make_uint2(pack2<F16>(v.x * inv, v.y * inv), pack2<F16>(v.z * inv, v.w * inv));
        if (c == 0) a.lse[row] = lse_of(mx, sum);
      } else {
        const long long at = (long long)job.part * a.parts.rows + row;
        *reinterpret_cast<float4*>(a.parts.o + at * D + c) = v;
        if (c == 0) a.parts.ml[at] = make_float2(mx, sum);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(s32(&sm.parts_read));
  }
  if (!a.first) settle_stream();
}

constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

// A row's parts in an order that follows from the row's own parts alone, whatever the other rows hold and however many pages its table has
// room for: part p belongs to the sum p % 8, whose parts are added up in turn, and the eight sums are joined in turn.  W warps share a row's
// sums out, sum s to warp s % W.  The lanes hold the parts' maxima and sums of weights, 32 at a time, and work out their factors.
//
// W follows from the most parts that any row can have, so that a warp takes what it asks for at once, or twice that (W = 8: in rounds of 64
// parts).  (us on the device, one and two warps for 9 to 16 parts: 1024 rows 108.8 and 106.7 a call; behind a prefix, where rows are
// many, 4096 rows 104.5 and 106.9: there one warp takes them by pairs of a sum, PAIRS.)  With eight warps a row, four parts a batch: eight
// spill, and where few of a wide table's pages are filled they cost 0.5 to 3 us of 13 to 103.
constexpr int kSums = 8;

template <int D, bool F16, int W, bool PAIRS>
__global__ void __launch_bounds__(kJoinThreads, 4) paged_join_kernel(const PagedGeo g, const PartsOut in, const View o, float* __restrict__ lse) {
  constexpr int V = D / 32, A = W == 8 ? 4 : 8;  // channels of a lane; parts that a warp asks for at a time
  constexpr int kHeld = W <= 2 ? 1 : 2;          // times 32 parts whose maxima stay in registers, and whose factors are worked out at once
  constexpr int kOwn = W == 1 ? 1 : kSums / W;   // sums that a warp has in registers
  constexpr int kRound = 32 * kHeld, kBatches = PAIRS || W >= 4 ? 2 : 1;  // parts of a round; batches that a warp takes of them
  static_assert(W == 8 ? kRound == A * W * kBatches : kRound >= A * W * kBatches, "rows of more parts have eight warps, and rounds");
  __shared__ alignas(16) float sums[W > 1 ? kJoinWarps / W : 1][kSums][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp % W;
  const int row = (int)blockIdx.x * (kJoinWarps / W) + warp / W;
  bool live = row < (int)in.rows;
  const int i = row % g.T, bh = row / g.T, b = live ? bh / g.H : 0, head = bh - b * g.H;
  const int zero = await_stream();
  const Parts p = parts_of(g, span_of(g, b + zero));
  live = live && i < p.ql;
  const int n = live ? in.shared + p.n : 0;
  const float2* ml = in.ml + row;
  const float* src = in.o + (long long)row * D + V * lane;
  const long long step = in.rows * D;
  // the warp's k-th part
  auto part_at = [&](int k) { return PAIRS ? (k >> 1) + kSums * (k & 1) : w + k * W; };
  float u[A][V];
  auto ask = [&](int k0) {
#pragma unroll
    for (int z = 0; z < A; ++z) {
      const float* at = src + min(part_at(k0 + z), n - 1) * step;
      if constexpr (V == 4) {
        const float4 t = __ldcg(reinterpret_cast<const float4*>(at));
        u[z][0] = t.x; u[z][1] = t.y; u[z][2] = t.z; u[z][3] = t.w;
      } else {
        const float2 t = __ldcg(reinterpret_cast<const float2*>(at));
        u[z][0] = t.x; u[z][1] = t.y;
      }
    }
  };
  auto read = [&](int y) { return y < n ? __ldcg(ml + y * in.rows) : make_float2(-INFINITY, 0.f); };
  float mx = -INFINITY, sum = 0.f, v[V], own[kOwn][V];
#pragma unroll
  for (int x = 0; x < V; ++x) {
    v[x] = 0.f;
#pragma unroll
    for (int s = 0; s < kOwn; ++s) own[s][x] = 0.f;
  }
  if (w < n) {  // (a warp without parts has nothing to add)
    float2 held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) held[k] = read(32 * k + lane);
    ask(0);
#pragma unroll
    for (int k = 0; k < kHeld; ++k) mx = fmaxf(mx, held[k].x);
    if constexpr (W == 8)
      for (int y = kRound + lane; y < n; y += 32) mx = fmaxf(mx, read(y).x);
#pragma unroll
    for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    int y0 = 0;
    do {
      float f[kHeld];
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const float2 part = y0 == 0 ? held[k] : read(y0 + 32 * k + lane);
        f[k] = part.x == -INFINITY ? 0.f : ex2(part.x - mx);
        sum += part.y * f[k];
      }
#pragma unroll
      for (int batch = 0; batch < kBatches; ++batch) {
        const int k0 = y0 / W + A * batch;
        if (batch > 0 || y0 > 0) {
          if (part_at(k0) >= n) break;
          ask(k0);
        }
#pragma unroll
        for (int z = 0; z < A; ++z) {
          const int at = part_at(k0 + z), in_round = part_at(A * batch + z);
          // (whether the part is one of the first 32 of the round does not depend on the warp)
          const float fz = __shfl_sync(0xffffffffu, f[kHeld == 1 || W * (A * batch + z) < 32 ? 0 : kHeld - 1], in_round & 31);
          float* to = own[W == 1 ? 0 : z % kOwn];
          if (at < n) {
#pragma unroll
            for (int x = 0; x < V; ++x) to[x] = fmaf(u[z][x], fz, to[x]);
          }
          if (W == 1 && (!PAIRS || z % 2)) {  // the sum is complete
#pragma unroll
            for (int x = 0; x < V; ++x) {
              v[x] = __fadd_rn(v[x], to[x]);
              to[x] = 0.f;
            }
          }
        }
      }
      y0 += kRound;  // (one warp's eight parts are one round; as a loop its loads stay ahead of the maxima: drafts in a window 24.3 -> 23.6 us)
    } while ((W == 8 || (W == 1 && !PAIRS)) && y0 < n);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int s = 0; s < kOwn; ++s) {
      float* to = &sums[warp / W][w + W * s][V * lane];
      if constexpr (V == 4) *reinterpret_cast<float4*>(to) = make_float4(own[s][0], own[s][1], own[s][2], own[s][3]);
      else *reinterpret_cast<float2*>(to) = make_float2(own[s][0], own[s][1]);
    }
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int s = 0; s < kSums; ++s)
#pragma unroll
      for (int x = 0; x < V; ++x) v[x] += sums[warp / W][s][V * lane + x];
  }
  if (!live) return;
  const float inv = inverse_of(sum);
  char* dst = o.data + b * o.sb + head * o.sh + i * o.sn + 2 * V * lane;
  if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<F16>(v[0] * inv, v[1] * inv), pack2<F16>(v[2] * inv, v[3] * inv));
  else *reinterpret_cast<uint32_t*>(dst) = pack2<F16>(v[0] * inv, v[1] * inv);
  if (lane == 0) lse[row] = lse_of(mx, sum);
}

// An item's weight beside its steps.  It takes as long as its keys take to arrive, 1260 cycles a step at D = 128 and 630 at 64, or, if that is
// longer, as one step takes from its keys to the end of the join: 3400 for one tile of 8 rows, 5300 for three, which is a whole chunk's
// time at D = 64, so that all items are alike there.  (us on the device with 2, and alike: 5 new tokens of 32 members, 12 heads on 3 of 64, 30.5
// and 26.8; 33 members with 4 behind a prefix 28.4 and 24.7.)
constexpr int turn_of(int d, int tiles) { return d == 128 ? 2 : tiles == 1 ? 4 : 0; }

template <int D, bool F16, int NT>
int launch_parts(const HostCtx& c, const PagedGeo& g, DecArgs a, const PoolMaps& maps, int most_parts) {
  constexpr size_t smem = sizeof(Smem<D, NT>) + 1024;
  static_assert(smem <= kMaxSmem, "more shared memory than a CTA can have");
  static unsigned long long configured = 0;
  int sms = 0;
  if (const int rc = launch_setup(reinterpret_cast<const void*>(paged_parts_kernel<D, F16, NT>), smem, &configured, &sms)) return rc;
  a.blocks = paged_row_blocks(D, g.G * g.T);
  const long long most = (long long)g.B * g.Hkv * a.blocks * most_parts;
  a.turn = turn_of(D, NT);
  return launch_kernel(paged_parts_kernel<D, F16, NT>, dim3((unsigned)(most < sms ? most : sms)), Smem<D, NT>::kThreads, smem, c.stream, true, 0, g, a, maps.k, maps.v);
}

template <int D, bool F16, int W, bool PAIRS = false>
int launch_join(const HostCtx& c, const PagedGeo& g, const PartsOut& parts, const View& o, float* lse) {
  constexpr int per = kJoinWarps / W;
  return launch_kernel(paged_join_kernel<D, F16, W, PAIRS>, dim3((unsigned)((parts.rows + per - 1) / per)), kJoinThreads, 0, c.stream, true, 0, g, parts, o, lse);
}

// Tiles of 8 rows that a CTA takes: what a step's accumulators leave room for in registers, and its sums in shared memory
int tiles_of(int d, int rows) { return rows <= 8 ? 1 : rows <= 16 || d == 128 ? 2 : rows <= 24 ? 3 : 4; }

// f(head dimension, type) as constants
template <class F>
int by_type(int d, bool f16, F&& f) {
  using std::integral_constant;
  if (d == 64) return f16 ? f(integral_constant<int, 64>{}, std::true_type{}) : f(integral_constant<int, 64>{}, std::false_type{});
  return f16 ? f(integral_constant<int, 128>{}, std::true_type{}) : f(integral_constant<int, 128>{}, std::false_type{});
}

}  // namespace

int paged_row_blocks(int d, int rows) {
  const int block = 8 * tiles_of(d, rows);
  return (rows + block - 1) / block;
}

bool paged_parts_fit(int d, int rows, long long units, int most_parts) {
  return units * paged_row_blocks(d, rows) * most_parts <= 0x7fffffffll / (kSteps + turn_of(d, tiles_of(d, rows)));
}

int launch_paged_parts(const HostCtx& c, const PagedGeo& g, bool f16, const View& q, const PoolMaps& maps, const PartsOut& parts,
                       int most_parts, bool direct, bool first, const View& o, float* lse) {
  const DecArgs a = {q, o, lse, parts, 0, maps.box_shift, 1, direct, first, 1.f / (float)g.G, c.status};
  return by_type(g.d, f16, [&](auto d, auto type) {
    constexpr int D = decltype(d)::value;
    constexpr bool F16 = decltype(type)::value;
    const int tiles = tiles_of(D, g.G * g.T);
    if constexpr (D == 64) {
      if (tiles == 4) return launch_parts<D, F16, 4>(c, g, a, maps, most_parts);
      if (tiles == 3) return launch_parts<D, F16, 3>(c, g, a, maps, most_parts);
    }
    return tiles == 2 ? launch_parts<D, F16, 2>(c, g, a, maps, most_parts) : launch_parts<D, F16, 1>(c, g, a, maps, most_parts);
  });
}

int launch_paged_join(const HostCtx& c, const PagedGeo& g, bool f16, const PartsOut& parts, int most_parts, const View& o, float* lse) {
  return by_type(g.d, f16, [&](auto d, auto type) {
    constexpr int D = decltype(d)::value;
    constexpr bool F16 = decltype(type)::value;
    if (most_parts <= 8) return launch_join<D, F16, 1>(c, g, parts, o, lse);
    if (most_parts <= 16) return parts.shared ? launch_join<D, F16, 1, true>(c, g, parts, o, lse) : launch_join<D, F16, 2>(c, g, parts, o, lse);
    return most_parts <= 64 ? launch_join<D, F16, 4>(c, g, parts, o, lse) : launch_join<D, F16, 8>(c, g, parts, o, lse);
  });
}

}  // namespace mosaic
