// Rows of query and key heads in a warp's registers, and their rotation by token index: what the kernels that turn heads share.
#pragma once
#include "common.cuh"

namespace mosaic {

namespace {

enum { kBf16 = 0, kF16 = 1, kF32 = 2 };
constexpr int kMaxHeadDim = 256;

// The helpers take a kernel's arguments (A), of which they read: d, channels of a head; rot, those that turn; lanes that a row is spread
// over; amplitude, factor of the turned channels.

template <int T>
struct Vec { static constexpr int n = T == kF32 ? 4 : 8, bytes = T == kF32 ? 4 : 2; };

template <int T>
__device__ __forceinline__ void widen(const uint4& v, float (&f)[Vec<T>::n]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (T == kF32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack16x2(w[i], T == kF16, f[2 * i], f[2 * i + 1]);
  }
}
template <int T>
__device__ __forceinline__ uint4 narrow(const float (&f)[Vec<T>::n]) {
  if constexpr (T == kF32) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  } else {
    return make_uint4(pack16x2(f[0], f[1], T == kF16), pack16x2(f[2], f[3], T == kF16), pack16x2(f[4], f[5], T == kF16),
                      pack16x2(f[6], f[7], T == kF16));
  }
}

// What a lane does in every row: its two pieces' channels, and the warp's share of rows.  Neighbouring lanes have neighbouring
// pieces, so that a load of either covers whole sectors.
struct Place {
  int ca, cb;         // first channel of either piece
  int group, groups;  // this lane's row of the `groups` rows that a warp takes at a time
  bool on;            // the lane has channels (d / 2V may be less than P)
};
template <int T, bool HALF, class A>
__device__ __forceinline__ Place place(const A& a, int lane) {
  constexpr int V = Vec<T>::n;
  Place p;
  const int slot = lane & (a.lanes - 1), turning = HALF ? a.rot / (2 * V) : 0, from = HALF ? a.rot : 0;
  p.on = slot * 2 * V < a.d;
  p.ca = slot < turning ? slot * V : from + (slot - turning) * V;
  p.cb = slot < turning ? a.rot / 2 + slot * V : from + (a.d - from) / 2 + (slot - turning) * V;
  p.group = lane / a.lanes;
  p.groups = 32 / a.lanes;
  return p;
}

// Cosines and sines of a token's angles, of all its pairs and V more; pairs that do not turn have (1, 0), which stand there from the start
constexpr int kAngles = kMaxHeadDim / 2 + 8;
struct Angles {
  float cosine[kAngles], sine[kAngles];
};
template <class A>
__device__ __forceinline__ void still_angles(const A& a, Angles& t, int lane) {
  for (int i = a.rot / 2 + lane; i < kAngles; i += 32) {
    t.cosine[i] = 1.f;
    t.sine[i] = 0.f;
  }
}
// The token's angles, shared out over the warp.  (`freqs`: behind the wait for the stream)
template <class A>
__device__ __forceinline__ void make_angles(const A& a, const double* freqs, long long pos, Angles& t, int lane) {
  __syncwarp();  // the token before has been read
  for (int i = lane; i < a.rot / 2; i += 32) {
    const double turns = (double)pos * (__ldg(freqs + i) * 0.31830988618379067154);  // half turns
    const float r = (float)(turns - 2.0 * rint(0.5 * turns));
    float sn, cn;
    sincospif(r, &sn, &cn);
    t.cosine[i] = cn * fabsf(a.amplitude);
    t.sine[i] = sn * a.amplitude;  // the launcher negates the factor to turn back
  }
  __syncwarp();
}
// N floats from an address that N floats align
template <int N>
__device__ __forceinline__ void read_floats(const float* p, float* out) {
  if constexpr (N == 2) {
    const float2 v = *reinterpret_cast<const float2*>(p);
    out[0] = v.x; out[1] = v.y;
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + j);
      out[j] = v.x; out[j + 1] = v.y; out[j + 2] = v.z; out[j + 3] = v.w;
    }
  }
}

// Turns the pairs of a row's two pieces.  (The angles are read anew for every row: kept over a token's rows they cost sixteen registers,
// which are worth a second CTA on the SM.)
__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
  const float u = x * c - y * s;
  y = x * s + y * c;
  x = u;
}
template <int V, bool HALF, class A>
__device__ __forceinline__ void turn_all(float (&a)[V], float (&b)[V], const Angles& t, const A& args, const Place& pl) {
  constexpr int N = HALF ? V : V / 2;  // pairs of one piece that lie side by side
  float c[V], s[V];
  const int i0 = HALF ? min(pl.ca, args.rot / 2) : pl.ca / 2;
  read_floats<N>(t.cosine + i0, c);
  read_floats<N>(t.sine + i0, s);
  if constexpr (!HALF) {
    read_floats<N>(t.cosine + pl.cb / 2, c + N);
    read_floats<N>(t.sine + pl.cb / 2, s + N);
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if constexpr (HALF) turn_pair(a[j], b[j], c[j], s[j]);
    else if (j < N) turn_pair(a[2 * j], a[2 * j + 1], c[j], s[j]);
    else turn_pair(b[2 * j - V], b[2 * j - V + 1], c[j], s[j]);
  }
}
// Neighbouring pairs of one piece, from channel `first` on
template <int V>
__device__ __forceinline__ void turn_piece(float (&f)[V], int first, const Angles& t) {
  float c[V / 2], s[V / 2];
  read_floats<V / 2>(t.cosine + first / 2, c);
  read_floats<V / 2>(t.sine + first / 2, s);
#pragma unroll
  for (int j = 0; j < V / 2; ++j) turn_pair(f[2 * j], f[2 * j + 1], c[j], s[j]);
}

// PART: some channels do not turn and stay as they are, whatever they hold.  (As pairs multiplied with (1, 0) an infinite one would
// make no number of its partner.)  With half pairs a lane's pairs turn, all of them, or none does; otherwise the border lies among the
// second pieces, or among the first and no second one turns.
template <int V, bool HALF, bool PART, class A>
__device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const Angles& t, const A& args, const Place& pl) {
  if constexpr (!PART) {
    turn_all<V, HALF>(a, b, t, args, pl);
  } else if constexpr (HALF) {
    if (pl.ca < args.rot / 2) turn_all<V, true>(a, b, t, args, pl);
  } else {
    auto border = [&](float (&f)[V], int first) {
      float g[V];
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] = f[j];
      turn_piece<V>(g, first, t);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = first + j < args.rot ? g[j] : f[j];
    };
    if (args.rot > args.d / 2) {
      turn_piece<V>(a, pl.ca, t);
      border(b, pl.cb);
    } else {
      border(a, pl.ca);
    }
  }
}
// The same on the two pieces as they lie in memory: what does not turn keeps its bits (narrowing would change those of what is no number).
template <int T, bool HALF, class A>
__device__ __forceinline__ void turn_part(uint4& va, uint4& vb, const Angles& t, const A& args, const Place& pl) {
  constexpr int V = Vec<T>::n;
  if constexpr (HALF) {
    if (pl.ca >= args.rot / 2) return;
    float a[V], b[V];
    widen<T>(va, a);
    widen<T>(vb, b);
    turn_all<V, true>(a, b, t, args, pl);
    va = narrow<T>(a);
    vb = narrow<T>(b);
  } else {
    auto turned = [&](const uint4& v, int first) {
      float f[V];
      widen<T>(v, f);
      turn_piece<V>(f, first, t);
      return narrow<T>(f);
    };
    auto border = [&](uint4& v, int first) {
      const uint4 u = turned(v, first);
      const int words = (args.rot - first) * Vec<T>::bytes / 4;  // that turn (a pair is one word or two)
      if (words > 0) v.x = u.x;
      if (words > 1) v.y = u.y;
      if (words > 2) v.z = u.z;
      if (words > 3) v.w = u.w;
    };
    if (args.rot > args.d / 2) {
      va = turned(va, pl.ca);
      border(vb, pl.cb);
    } else {
      border(va, pl.ca);
    }
  }
}

}  // namespace

}  // namespace mosaic
