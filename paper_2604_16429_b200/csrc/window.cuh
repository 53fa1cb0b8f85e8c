// Geometry of the sliding-window attention shared by its kernels.
#pragma once
#include "tc_common.cuh"

namespace mosaic {

constexpr int kMaxSinks = 128;
constexpr int kRows = 128;  // rows of a query or key tile (the M of one tensor-core product)

struct WinGeo {
  int B, H, Hkv, G;       // G = H / Hkv query heads share a key/value head
  int Nq, Nk, d;
  int window, sinks;      // both at most Nk
  float scale, scale_log2;
  const int32_t *q_len, *k_len;
};

// Lengths of batch member b: its queries are the last ql of its kl tokens
struct Span {
  int ql, kl, off;  // row i has position off + i
};
__device__ __forceinline__ Span span_of(const WinGeo& g, int b) {
  Span s;
  s.ql = g.q_len ? min(max(__ldg(g.q_len + b), 0), g.Nq) : g.Nq;
  s.kl = g.k_len ? min(max(__ldg(g.k_len + b), 0), g.Nk) : g.Nk;
  s.off = s.kl - s.ql;
  return s;
}

// The bounded waits without a call: the registers of a warpgroup that raised or lowered its count would all be saved around one
// (2 KB of stack and as many spills a thread in the forward).
__device__ __forceinline__ bool wait_here(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
#pragma unroll 1
  for (uint32_t i = 1;; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 63u) == 0u) {
      if (*abort) return false;
      if (clock64() - t0 > kSpinCycles) {
        set_status(status, MOSAIC_E_DEVICE_TIMEOUT);
        *abort = 1;
        return false;
      }
    }
  }
}
__device__ __forceinline__ bool warp_wait_here(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
  return __all_sync(0xffffffffu, wait_here(bar, parity, abort, status));
}

// The lowest n bits (n any integer)
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// `bytes` (a multiple of 16, both ends aligned) of global memory to shared memory
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar)
               : "memory");
}

// Operand descriptors.  A tile of R rows by d channels lies in d/64 parts of R x 64 channels (128-byte swizzled rows), `part`
// bytes apart.  K-major operand (contraction over channels): the descriptor of 16 channels at 16 kk.  MN-major operand
// (contraction over rows, all d channels side by side): the descriptor of rows 16 kk .. 16 kk + 15, its 64-channel groups `part` apart.
__device__ __forceinline__ uint64_t k_major(uint64_t tile, int kk, uint32_t part) {
  return tile + (uint64_t)(((kk >> 2) * part + (kk & 3) * 32) >> 4);
}
__device__ __forceinline__ uint64_t mn_major(uint32_t addr, uint32_t part) {
  return (smem_desc(addr) & ~((uint64_t)0x3fff << 16)) | ((uint64_t)(part >> 4) << 16);
}
__device__ __forceinline__ uint32_t idesc_n(uint32_t base, int n) { return base | ((uint32_t)(n >> 3) << 17); }

// Rows first .. R - 1 of a tile to zero (rows that do not exist may hold anything, and a weight of zero does not silence a NaN),
// by a whole warp; visible to the tensor core afterwards.
template <int D>
__device__ __forceinline__ void zero_rows(unsigned char* tile, int first, int rows, int lane) {
  for (int r = max(first, 0); r < rows; ++r)
    if (lane < D / 8) *reinterpret_cast<uint4*>(tile + (lane >> 3) * rows * 128 + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}

int make_win_geo(const mosaic_window_params* p, const int32_t* q_len, const int32_t* k_len, WinGeo* g);

// launch_setup for a kernel whose warpgroups share out `regs` registers a thread anew: refused if the compiler gave it another
// number, because the increase would then wait for registers that nobody has.  (`done` as there.)
inline int launch_setup_regs(const void* func, int regs, size_t smem, unsigned long long* done, int* sms) {
  const unsigned long long before = *done;
  const int rc = launch_setup(func, smem, done, sms);
  if (rc || *done == before) return rc;
  cudaFuncAttributes at;
  if (cudaFuncGetAttributes(&at, func) != cudaSuccess) { *done = before; return MOSAIC_E_CUDA; }
  if (at.numRegs != regs) { *done = before; return MOSAIC_E_UNSUPPORTED; }
  return MOSAIC_OK;
}

// Views whose heads or members all lie at one place (stride 0) have a map with one of them.
struct Fold {
  int h, b;  // factor of the head's and the member's coordinate
};
inline Fold fold_of(const View& v) { return {v.sh ? 1 : 0, v.sb ? 1 : 0}; }

int launch_window_fwd(const HostCtx& c, const WinGeo& g, bool f16, const View& q, const View& k, const View& v, const View& o,
                      float* lse);
struct WinBwd {
  View q, k, v, o, d_o, dq, dk, dv;
  const float* lse;
};
struct WinBwdWs {
  size_t neg_lse2, neg_d, partial, total;
  int pad, pieces, piece_rows;
};
WinBwdWs window_bwd_layout(const WinGeo& g);
int launch_window_bwd(const HostCtx& c, const WinGeo& g, bool f16, const WinBwd& t, void* ws);
int launch_window_decode(const HostCtx& c, const WinGeo& g, bool f16, int ring, const View& q, const View& k, const View& v,
                         const View& o, float* lse);

}  // namespace mosaic
