// Rotary positions of several axes on the packed projection [b*s, 3h], in place.
//
// A head's first 2 n elements are n pairs (p, q).  Pair i belongs to an axis x(i) (time, height, width, ...) and turns by the angle
// t = pos[x(i)][token] * freq(i):  p' = p cos t - q sin t,  q' = q cos t + p sin t;  the backward pass turns the gradient by -t.  The
// angle depends on the token and the pair only, so the 2 a heads of a token's Q and K share one table of n (cos, sin).
//
// 2/3 of the projection is read and written once: bound by memory where it is large (2048 tokens x 64 heads of 128 in bf16: 21.4 us and 6.3 TB/s a
// launch on the same tensors again, whose lines the memory-side cache holds in part, 27.6 on others), by the latency of a workgroup's life (loads,
// table, stores) where it is small: waves wait 2/3 to 3/4 of their time (profiles/operators_counters.txt).
// A workgroup takes as many whole tokens as give its 256 threads U vectors each, or a part of one; it asks for its vectors first, and makes the table in
// LDS while they are on their way.  U: 1 for 16-byte vectors of both halves in bf16, whose 32 registers a piece cost waves, 3 otherwise.  Two launches,
// there and back, over U: 2048 tokens x 64 heads of 128 58 | 65 us with 1 | 4; one: 4 x 1024 x 16 heads of 96, fp32 22.0 | 20.1 | 21.3 with 1 | 3 | 4,
// bf16 neighbours 14.2 | 10.0 | 10.5.  Whole tokens leave places idle (288 vectors a token: 576 of 768).  Angles are taken in turns
// (freq / 2 pi), in 64 bits, and reduced to [-1/2, 1/2] there: a float has no fraction left at position 10^6.  What a float loses of the reduced angle
// is put back into its sine and cosine, or that error would be as large as their own rounding (cosines off by 3.4e-8 rms instead of 1.9e-8, in the same time).
#include <cmath>

#include "kernels.hpp"

namespace k2bw {
namespace {

constexpr int kRotMaxPairs = 64, kRotThreads = 256, kRotMaxTokens = 32;
template <typename T, int V, bool HALF> constexpr int kRotPerThread = HALF && V == 8 ? 1 : 3;

struct RotaryParams {
  void* x;
  const int32_t* pos;      // [axes][tokens], or null: the token's place in its sequence
  int64_t tokens;
  int s, row, dh, n, heads2, per_group, parts;   // row: elements of a row; heads2: heads of Q and K; per_group: tokens of a workgroup; parts: workgroups of a token
  int inverse;
  uint8_t axis[kRotMaxPairs];
  double turns[kRotMaxPairs];   // freq / 2 pi
};

// V consecutive elements as they lie in memory
template <typename T, int V> struct RawOf;
template <> struct RawOf<float, 4> { using type = uint4; };
template <> struct RawOf<float, 2> { using type = uint2; };
template <> struct RawOf<float, 1> { using type = uint32_t; };
template <> struct RawOf<bf16_t, 8> { using type = uint4; };
template <> struct RawOf<bf16_t, 4> { using type = uint2; };
template <> struct RawOf<bf16_t, 2> { using type = uint32_t; };
template <> struct RawOf<bf16_t, 1> { using type = uint16_t; };

template <typename T, int V>
__device__ __forceinline__ void unpack(const typename RawOf<T, V>::type& raw, float (&v)[V]) {
  T e[V];
  __builtin_memcpy(e, &raw, sizeof raw);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = Act<T>::load(e + i);
}
template <typename T, int V>
__device__ __forceinline__ typename RawOf<T, V>::type pack(const float (&v)[V]) {
  T e[V];
#pragma unroll
  for (int i = 0; i < V; ++i) Act<T>::store(e + i, v[i]);
  typename RawOf<T, V>::type raw;
  __builtin_memcpy(&raw, e, sizeof raw);
  return raw;
}

// V: elements per access; a thread turns V pairs (HALF: elements i and i + n) or V / 2 (neighbours 2i and 2i + 1).
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryParams p) {
  using Raw = typename RawOf<T, V>::type;
  constexpr int P = HALF ? V : V / 2;   // pairs per vector
  constexpr int U = kRotPerThread<T, V, HALF>, kItems = kRotThreads * U;
  __shared__ float2 table[kRotMaxTokens * kRotMaxPairs];
  const int part = blockIdx.x % p.parts;   // of a token
  const int64_t t0 = (int64_t)(blockIdx.x / p.parts) * p.per_group;
  const int toks = (int)min((int64_t)p.per_group, p.tokens - t0);
  const int nv = p.n / P, items = p.heads2 * nv, total = min(toks * items, (part + 1) * kItems);
  T* base = static_cast<T*>(p.x) + t0 * p.row;
  const int e0 = part * kItems + threadIdx.x;
  // A thread's (first) angle is asked for in front of its vectors: loads come back in order, and it has the longer way to go.
  auto angle = [&](int e, double& turns) __attribute__((always_inline)) {
    const int tok = e / p.n, i = e - tok * p.n;
    const int64_t t = t0 + tok;
    turns = p.turns[i];
    return p.pos ? p.pos[p.axis[i] * p.tokens + t] : (int)(t % p.s);
  };
  int pos = 0;
  double turns = 0.0;
  if ((int)threadIdx.x < toks * p.n) pos = angle(threadIdx.x, turns);
  Raw lo[U], hi[U];
  T* at[U];
  int entry[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = e0 + u * kRotThreads;
    if (e < total) {
      const int tok = e / items, r = e - tok * items, head = r / nv, v = r - head * nv;
      entry[u] = tok * p.n + v * P;
      at[u] = base + (int64_t)tok * p.row + head * p.dh + v * V;
      lo[u] = *reinterpret_cast<const Raw*>(at[u]);
      if (HALF) hi[u] = *reinterpret_cast<const Raw*>(at[u] + p.n);
    }
  }
  for (int e = threadIdx.x; e < toks * p.n; e += kRotThreads) {
    if (e >= kRotThreads) pos = angle(e, turns);
    const double turn = (double)pos * turns, half = 2.0 * (turn - rint(turn));
    const float near = (float)half, rest = (float)(half - (double)near) * 3.14159265f;   // (what the rounding to 24 bits takes from the angle, to first order)
    float sn, cs;
    sincospif(near, &sn, &cs);
    const float c1 = fmaf(-rest, sn, cs), s1 = fmaf(rest, cs, sn);
    table[e] = make_float2(c1, p.inverse ? -s1 : s1);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (e0 + u * kRotThreads < total) {
      float a[V];
      unpack<T, V>(lo[u], a);
      if constexpr (HALF) {
        float b[V], x[V], y[V];
        unpack<T, V>(hi[u], b);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float2 cs = table[entry[u] + j];
          x[j] = a[j] * cs.x - b[j] * cs.y;
          y[j] = b[j] * cs.x + a[j] * cs.y;
        }
        *reinterpret_cast<Raw*>(at[u]) = pack<T, V>(x);
        *reinterpret_cast<Raw*>(at[u] + p.n) = pack<T, V>(y);
      } else {
        float x[V];
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const float2 cs = table[entry[u] + j];
          x[2 * j] = a[2 * j] * cs.x - a[2 * j + 1] * cs.y;
          x[2 * j + 1] = a[2 * j + 1] * cs.x + a[2 * j] * cs.y;
        }
        *reinterpret_cast<Raw*>(at[u]) = pack<T, V>(x);
      }
    }
  }
}

template <typename T, int V, bool HALF>
hipError_t launch_rotary(RotaryParams p, hipStream_t s) {
  const int items = p.heads2 * (p.n / (HALF ? V : V / 2));
  constexpr int kItems = kRotThreads * kRotPerThread<T, V, HALF>;
  p.per_group = kItems / items;
  if (p.per_group < 1) p.per_group = 1;
  if (p.per_group > kRotMaxTokens) p.per_group = kRotMaxTokens;
  p.parts = items > kItems ? (items + kItems - 1) / kItems : 1;
  const int64_t groups = (p.tokens + p.per_group - 1) / p.per_group * p.parts;
  if (groups * kRotThreads > kMaxThreads) return hipErrorInvalidValue;
  hipLaunchKernelGGL((rotary_kernel<T, V, HALF>), dim3((unsigned)groups), dim3(kRotThreads), 0, s, p);
  return hipGetLastError();
}

// The widest access that the pairs' places allow: heads start at multiples of 8 elements, the second halves n further on.
template <typename T>
hipError_t pick_rotary(const RotaryParams& p, bool half, hipStream_t s) {
  constexpr int W = Act<T>::kVec;
  if (half) {
    if (p.n % W == 0) return launch_rotary<T, W, true>(p, s);
    if (p.n % (W / 2) == 0) return launch_rotary<T, W / 2, true>(p, s);
    if (W == 8 && p.n % 2 == 0) return launch_rotary<T, 2, true>(p, s);
    return launch_rotary<T, 1, true>(p, s);
  }
  if (p.n % (W / 2) == 0) return launch_rotary<T, W, false>(p, s);
  if (W == 8 && p.n % 2 == 0) return launch_rotary<T, 4, false>(p, s);
  return launch_rotary<T, 2, false>(p, s);
}

}  // namespace

hipError_t rotary(const RotaryDesc& d, void* x, hipStream_t stream) {
  if (d.b <= 0 || d.s <= 0 || d.a <= 0 || d.dh <= 0 || d.dh % 8 || d.dh > 2 * kRotMaxPairs) return hipErrorInvalidValue;
  if (d.n_pairs < 1 || 2 * d.n_pairs > d.dh || d.pairing < 0 || d.pairing > 1 || !d.axis_of_pair || !d.freq || d.n_axes < 1 || d.n_axes > 255)
    return hipErrorInvalidValue;
  if (!x || (reinterpret_cast<uintptr_t>(x) & 15) || (reinterpret_cast<uintptr_t>(d.pos) & 3)) return hipErrorInvalidValue;
  if ((int64_t)3 * d.a * d.dh > (1 << 30)) return hipErrorInvalidValue;
  RotaryParams p{};
  p.x = x; p.pos = d.pos; p.tokens = (int64_t)d.b * d.s; p.s = d.s; p.row = 3 * d.a * d.dh; p.dh = d.dh; p.n = d.n_pairs;
  p.heads2 = 2 * d.a; p.inverse = d.inverse ? 1 : 0;
  for (int i = 0; i < d.n_pairs; ++i) {
    if (d.axis_of_pair[i] >= d.n_axes || !(std::fabs(d.freq[i]) <= 0x1p900)) return hipErrorInvalidValue;   // (positions times it: finite)
    p.axis[i] = d.axis_of_pair[i];
    p.turns[i] = d.freq[i] / 6.283185307179586476925286766559;
  }
  if (d.dtype == kBF16) return pick_rotary<bf16_t>(p, d.pairing == 0, stream);
  if (d.dtype == kF32) return pick_rotary<float>(p, d.pairing == 0, stream);
  return hipErrorInvalidValue;
}

}  // namespace k2bw
