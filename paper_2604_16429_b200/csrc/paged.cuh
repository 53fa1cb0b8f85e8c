// Geometry of the paged cache shared by the kernels that write and read it.
#pragma once
#include "window.cuh"

namespace mosaic {

constexpr int kMinPage = 16;    // slots of a page at least: 16 keys, the rows of one product, never leave one
constexpr int kMaxPage = 1 << 20;
constexpr int kMaxNew = 16;     // new tokens a sequence that the attention takes
constexpr int kChunkKeys = 512; // keys whose attention is one part, joined with the others at the end
constexpr int kSms = 148;       // of the device that the kernels are built for

// A pool of pages and the table that says which of them hold a member's tokens: token j lies in slot j % page of page
// table[b][j / page].
struct PagedGeo {
  int B, H, Hkv, G, T, d;  // T: rows of q a member
  int shift, pages, width; // log2 of a page's slots; pages of the pool; entries of a table row
  int window, sinks;       // window 0: none
  long long table_stride;
  const int32_t *table, *k_len, *q_len;
  float scale_log2;
};

// Lengths of member b: its new tokens are the last ql of its kl
__device__ __forceinline__ Span clamped(const PagedGeo& g, int k_len, int q_len) {
  Span s;
  s.ql = min(max(q_len, 0), g.T);
  s.kl = min(max(k_len, 0), g.width << g.shift);
  s.off = s.kl - s.ql;
  return s;
}
__device__ __forceinline__ Span span_of(const PagedGeo& g, int b) {
  return clamped(g, __ldg(g.k_len + b), g.q_len ? __ldg(g.q_len + b) : g.T);
}

// The keys that member b's rows see, cut into parts: the chunks of kChunkKeys positions that hold some of them.  So what a part is
// follows from positions alone, and a row's bits depend neither on what else is in the call nor on its table's width (the join keeps to
// that).
struct Parts {
  int kl, ql, p0;   // tokens, new ones, position of the first row
  int from, sinks;  // the rows see keys of [0, sinks) and of [from, kl) only
  int first, front; // chunk of `from`; 1: the sinks lie in a chunk ahead of it, the first part
  int n;            // parts
};
__device__ __forceinline__ Parts parts_of(const PagedGeo& g, const Span& s) {
  Parts p;
  p.kl = s.kl; p.ql = s.ql; p.p0 = s.off;
  p.from = g.window ? max(0, s.off - g.window + 1) : 0;
  p.sinks = g.window ? min(g.sinks, s.kl) : 0;
  p.first = p.from / kChunkKeys;
  p.front = p.sinks > 0 && p.first > 0;
  p.n = s.kl > 0 && s.ql > 0 ? (s.kl - 1) / kChunkKeys - p.first + 1 + p.front : 0;
  return p;
}
// Chunk of part o
__device__ __forceinline__ int chunk_of(const Parts& p, int o) { return p.front ? (o ? p.first + o - 1 : 0) : p.first + o; }

// What parts leave for the join, in the workspace: the rows' weighted sums of values [part][row][d], their maximum (base 2, scaled) and
// sum of weights [part][row], fp32; rows are [B, H, T].  The prefix' parts come first, then the member's own.
struct PartsOut {
  float* o;
  float2* ml;
  long long rows;
  int shared;  // parts of the prefix
};

// The two halves of await_stream, for a kernel that does not read what the one ahead of it writes: it lets the next kernel in at its
// start, works on what was complete when the one ahead began, and waits for that one before it ends, so that the chain holds.
__device__ __forceinline__ int pass_stream() {
  int zero;
  asm volatile("griddepcontrol.launch_dependents;\n\tmov.u32 %0, 0;" : "=r"(zero) : : "memory");
  return zero;
}
__device__ __forceinline__ void settle_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// A pool as a tensor [pages, Hkv, page, d], strides in bytes
int check_pool(const mosaic_view* v, const mosaic_paged_params* p, View* out);

struct AppendTensors {
  View q, q_out, k, v, k_pages, v_pages;
};
int launch_paged_append(const HostCtx& c, const PagedGeo& g, const mosaic_paged_params* p, const double* freqs, const AppendTensors& t);

// A map of a pool in boxes of `rows` slots by `parts` times 64 channels, and the copy of one from 64 * part on
bool make_map_pool(CUtensorMap* map, const View& v, int d, int page, int heads, int pages, int rows, int parts);
__device__ __forceinline__ void load_slots(uint32_t dst, const CUtensorMap* map, uint32_t bar, int slot, int part, int head, int page) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(slot), "r"(part), "r"(head), "r"(page)
      : "memory");
}
constexpr int kBoxShift = 6;  // log2 of the slots that a box has at the most: the keys of a step

// The pools and their maps in boxes of a page, or of a step's slots, and all channels
struct PoolMaps {
  View k_pages, v_pages;
  CUtensorMap k, v;
  int box_shift;  // log2 of a box's slots
  bool make(const PagedGeo& g) {
    box_shift = g.shift < kBoxShift ? g.shift : kBoxShift;
    return make_map_pool(&k, k_pages, g.d, 1 << g.shift, g.Hkv, g.pages, 1 << box_shift, g.d / 64) &&
           make_map_pool(&v, v_pages, g.d, 1 << g.shift, g.Hkv, g.pages, 1 << box_shift, g.d / 64);
  }
};

// Blocks that the rows of a key/value head are taken in
int paged_row_blocks(int d, int rows);
// Whether the list of all items can be counted: `units` key/value heads of all members, `rows` of each, in `most_parts` parts
bool paged_parts_fit(int d, int rows, long long units, int most_parts);
// Attention over the members' own pages: parts to the workspace, or, where a member can have but one, results (`direct`), joined with the
// prefix' parts if there are any.  `first`: the call's first kernel, which clears the status word; otherwise it follows the prefix' kernel.
int launch_paged_parts(const HostCtx& c, const PagedGeo& g, bool f16, const View& q, const PoolMaps& maps, const PartsOut& parts,
                       int most_parts, bool direct, bool first, const View& o, float* lse);
// Attention over a prefix that all members share: its parts are the first of every row.  How it is cut follows from its length, the
// key/value heads and the rows of a head; `chunk`: keys of a part.
int prefix_parts(int len, int kv_heads, long long rows, int* chunk);
int launch_prefix_fwd(const HostCtx& c, const PagedGeo& g, bool f16, const View& q, const PoolMaps& maps, const int32_t* prefix_table,
                      int prefix_len, int chunk, const PartsOut& parts);
// Joins all parts of every row
int launch_paged_join(const HostCtx& c, const PagedGeo& g, bool f16, const PartsOut& parts, int most_parts, const View& o, float* lse);

}  // namespace mosaic
