// Orthogonalised updates: the Newton-Schulz iteration X <- P(A) X, P(A) = a I + b A + c A^2, A = X X', from X = U / |U| (Frobenius norm),
// for a batch of matrices of one size, and the optimizer step made of it.
//
// The matrices are worked on in the wide form (m rows <= n columns; a tall one is transposed on its way in and out), padded with zeros to
// multiples of 64.  An m x m matrix M is held as its mean eigenvalue and the rest: M = mean I + M', mean = tr(M) / m.  M' and X are sums of
// two fp16 numbers (hi + lo, 22 bits); the matrix cores multiply the fp16 parts, everything linear takes both:
//   L R = mean_L mean_R I + mean_R L' + mean_L R' + L' R',    X <- mean_P X + P' X.
// What the matrices are on average never passes through 11 bits that way, and X is only rounded where it is multiplied by a P' of mean
// zero.  Off the 64-bit result after five default steps (2-norm): 2e-4 to 2e-3 (the most for small ranks and little else), a bf16 result's own
// rounding being 1.7e-3, and up to 1e-2 where a few rows or directions are more than a hundred times the others; with fp16 numbers for all of A, P
// and X 4e-4 to 2e-2, with bf16 1e-2 to 1.7e-1.  fp32 results take three products, hi hi + hi lo + lo hi: 3e-7 to 2e-4, 0.04 to 1 times what the
// iteration in 32-bit arithmetic is off by on this card (2.3 times, 1.1e-6, beside one row that is 300 times the others), at three times the matrix
// time, where the fp32 matrix instructions take sixteen.  A K tile holds both
// planes of either operand and gives all three (gemm_lds.hpp's PLANES): operands arrive at about 36 bytes a cycle and CU in every shape, and the
// products one after the other, of planes fetched three times, take 1.05 (2560 x 10240) to 1.24 (943 x 3768) of the time.
//
// The first two steps together where X is wide: A_1 = X_1 X_1' = P_1 A_0 P_1 needs no pass over X, and X_2 = (P_2 P_1) X_0 only one, so they cost
//   gram A_0 (half of 2 m^2 n: symmetric), P_1, U = A_0 P_1, A_1 = U P_1, P_2, Q = P_2 P_1 (half of 2 m^3 each), X <- Q X (2 m^2 n)
// against twice gram, P, X <- P X: 3 n + 5 m against 6 n + 2 m times m^2.  What A_0 is off by grows by a^2 on the smallest singular values; in front
// the single steps behind divide it out again as those values grow, further back they do not.  1024 x 4096 | 1536 x 4608 of rank m/4 and 1 % noise, with
// two, one, two together: bf16 results off by 7.1e-3 | 7.3e-3, so 1.9e-3 | 1.9e-3 (1.7e-3 of it rounding; 1.0e-3 is what single steps are off by before
// it).  fp32, three and two together 7.0e-6 | 1.5e-5, so 4.5e-6 | 4.5e-6, the 32-bit iteration 8.7e-6 | 8.3e-6.  Three in front, fp32: up to 6 times that
// beside one row that is 300 times the others.
//
// The means are sums of products of entries that the epilogues leave per tile and that whoever needs them adds up in one order, so
// results do not depend on timing.  They are shifts that drop out of the polynomial: their own rounding does not matter.
#include <algorithm>
#include <cmath>

#include "gemm_lds.hpp"
#include "kernels.hpp"

namespace k2bw {
namespace {

constexpr int kPad = 64;
// Powers of two that the fp16 numbers are kept at.  X has entries of at most about 1.2 (its singular values' bound) and of 1 / sqrt(m n) to
// begin with; A and A P of at most 1.5; P and P P of at most a^2 = 12.
constexpr float kScaleX = 4096.f, kScaleA = 4096.f, kScaleP = 1024.f;

enum Product : int { kGram = 0, kMul = 1, kUpdate = 2, kLast = 3 };   // X X'; L R of two m x m matrices; X <- P X; the same to where X leaves for

struct OrthProduct {
  const bf16_t *A, *B;                               // of matrix 0; as BfParams and TileWalk name things
  int M, N, K, lda, ldb;
  int seg_tiles;                                     // all K tiles, in tiles of the kernel's own K
  uint32_t a_seg, b_seg, a_stride256, b_stride256;   // (one piece: 0)
  uint32_t a_plane, b_plane;                         // PLANES: bytes from an operand's hi to its lo
  int64_t matrix;                                    // bytes from one matrix's part of the workspace to the next
  bf16_t* out; int ldo; int64_t out_plane;           // planes in elements
  const bf16_t *left, *right; int64_t old_plane;     // the operands' entries for the linear part (kUpdate: left = X), row length ldo
  int with; const bf16_t* partner;                   // sums_out: of out times out (0), left (1), right (2) or partner (3)
  const float* sums_in; int n_sums; float* sums_out;
  float* means; int mean_left, mean_right, mean_out; // places in `means`
  int poly;                                          // kMul: right = left, and the result is a + b L + c L^2
  float a, b, c, inv_m, scale_left, scale_right, scale_out;
  int m, tiles, tiles_n, total;                      // m: rows that are not padding; tiles of a matrix, of the launch
  int first;                                         // kGram: X still has norm 1
  int whole;                                         // a symmetric result in all of its tiles: nothing is mirrored
};

// The caller's matrices: element (i, r, c) at i * stride + r * ld + c.
enum End : int { kEndF32 = 0, kEndBf16 = 1, kEndMuon = 2 };
struct OrthEnds {
  int kind;
  const void* in; void* out;             // orthogonalize: fp32 or bf16
  int64_t in_stride, out_stride; int ld_in, ld_out;
  // muon: all fp32 with in_stride and ld_in
  const float *w, *G; float *w_next, *m; bf16_t* w_lp;
  float lr, beta, omb, keep, inv_micro;  // lr: times the scale; omb: 1 - beta; keep: 1 - lr * decay
  int nesterov;
  int rows, cols;
  bool tall;
  bf16_t* X; int64_t plane, matrix; int ldx;   // the padded copy: elements, elements, bytes
  double* squares; int n_squares;        // [matrix][n_squares] in the matrix's part
};

// 8 neighbours of a row leave: x as it is, or into the weights w (read ahead).
__device__ __forceinline__ void orth_leave(const OrthEnds& e, int matrix, int r, int c, const float (&x)[8], const float (&w)[8]) {
  if (e.kind == kEndMuon) {
    const int64_t at = matrix * e.in_stride + (int64_t)r * e.ld_in + c;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = w[j] * e.keep - e.lr * x[j];
    store8(e.w_next + at, v);
    if (e.w_lp) store8(e.w_lp + at, v);
  } else {
    const int64_t at = matrix * e.out_stride + (int64_t)r * e.ld_out + c;
    if (e.kind == kEndBf16) store8(static_cast<bf16_t*>(e.out) + at, x);
    else store8(static_cast<float*>(e.out) + at, x);
  }
}
struct NoEnds {};
template <int KIND> struct EndsOf { using type = NoEnds; };
template <> struct EndsOf<kLast> { using type = OrthEnds; };

__device__ __forceinline__ uint16_t f16_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ float f16_float(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
__device__ __forceinline__ void unpack_f16x8(const uint4& w, float (&v)[8]) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = f16_float((uint16_t)x[i]); v[2 * i + 1] = f16_float((uint16_t)(x[i] >> 16)); }
}
__device__ __forceinline__ void load_f16x8(const bf16_t* p, float (&v)[8]) { unpack_f16x8(*reinterpret_cast<const uint4*>(p), v); }
__device__ __forceinline__ uint4 pack_f16x8(const uint16_t (&e)[8]) {
  return make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
}
// value -> its two fp16 numbers
__device__ __forceinline__ void split8(const float (&r)[8], uint16_t (&hi)[8], uint16_t (&lo)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) { hi[j] = f16_bits(r[j]); lo[j] = f16_bits(r[j] - f16_float(hi[j])); }
}

// A symmetric result is computed in the tiles that touch the lower triangle; an entry is mirrored where its image lies in no such tile.
template <int BM, int BN>
__host__ __device__ constexpr bool in_lower_tile(int row, int col) { return row / BM * BM + BM - 1 >= col / BN * BN; }

// The matrix and tile of a workgroup: consecutive tiles to an XCD's workgroups.
struct OrthPlace { int matrix, bm, bn, tile; };
template <int KIND, int BM, int BN>
__device__ __forceinline__ OrthPlace orth_place(const OrthProduct& p) {
  const int b = blockIdx.x, whole = p.total / 8 * 8;
  const int id = b < whole ? (b & 7) * (p.total / 8) + (b >> 3) : b;
  OrthPlace o;
  o.matrix = id / p.tiles;
  o.tile = id - o.matrix * p.tiles;
  if (KIND >= kUpdate) {
    // (as tile_coords in gemm_bf16.hip: groups of 8 tile rows, column by column)
    const int tiles_m = p.tiles / p.tiles_n, per_group = 8 * p.tiles_n, group = o.tile / per_group, first = group * 8;
    const int gm = min(8, tiles_m - first), in = o.tile - group * per_group;
    o.bm = first + in % gm;
    o.bn = in / gm;
  } else if (p.whole) {
    o.bm = o.tile / p.tiles_n;
    o.bn = o.tile - o.bm * p.tiles_n;
  } else {   // row by row
    int row = 0, left = o.tile;
    for (;; ++row) {
      const int n = min(p.tiles_n, (row * BM + BM - 1) / BN + 1);
      if (left < n) break;
      left -= n;
    }
    o.bm = row;
    o.bn = left;
  }
  return o;
}

// What a launch's epilogue makes of the products' sums x: f1 L + f2 R + f3 x - (diagonal ? shift : 0), all as they are kept; and the mean.
struct OrthFactors { float f1, f2, f3, shift, mean; };
template <int KIND>
__device__ __forceinline__ OrthFactors orth_factors(const OrthProduct& p, float sum, float left, float right) {
  if (KIND >= kUpdate) return {left, 0.f, 1.f / p.scale_left, 0.f, 0.f};
  if (KIND == kGram) {
    const float mean = p.first ? p.inv_m : sum * (p.inv_m / (kScaleX * kScaleX));
    return {0.f, 0.f, p.scale_out / (kScaleX * kScaleX), mean * p.scale_out, mean};
  }
  const float t = sum * (p.inv_m / (p.scale_left * p.scale_right)), f3 = p.scale_out / (p.scale_left * p.scale_right);
  if (p.poly) return {(p.b + 2.f * p.c * left) * (p.scale_out / p.scale_left), 0.f, p.c * f3, p.c * t * p.scale_out, p.a + p.b * left + p.c * (left * left + t)};
  return {right * (p.scale_out / p.scale_left), left * (p.scale_out / p.scale_right), f3, t * p.scale_out, left * right + t};
}

// What the epilogue reads for 8 neighbours of a row, asked for ahead of its use.
template <int KIND> struct OrthOld { uint4 l[2], r[2], partner; };
template <> struct OrthOld<kUpdate> { uint4 l[2]; };
template <> struct OrthOld<kLast> { uint4 l[2]; float w[8]; };
template <> struct OrthOld<kGram> {};
template <int KIND>
__device__ __forceinline__ void orth_ask(const OrthProduct& p, int64_t skip, int row, int col, OrthOld<KIND>& o) {
  if constexpr (KIND != kGram) {
    const int64_t at = skip + (int64_t)row * p.ldo + col;
    o.l[0] = *reinterpret_cast<const uint4*>(p.left + at);
    o.l[1] = *reinterpret_cast<const uint4*>(p.left + p.old_plane + at);
    if constexpr (KIND == kMul) {
      if (!p.poly) {
        o.r[0] = *reinterpret_cast<const uint4*>(p.right + at);
        o.r[1] = *reinterpret_cast<const uint4*>(p.right + p.old_plane + at);
      }
      if (p.with == 3) o.partner = *reinterpret_cast<const uint4*>(p.partner + at);
    }
  }
}
// The finished values, and the sum of their products with the partner's.
template <int KIND>
__device__ __forceinline__ float orth_finish(const OrthProduct& p, const OrthFactors& f, int row, int col, const OrthOld<KIND>& o, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = v[j] * f.f3 - (KIND < kUpdate && row == col + j && row < p.m ? f.shift : 0.f);
  if constexpr (KIND != kGram) {
    float hi[8], lo[8];
    unpack_f16x8(o.l[0], hi);
    unpack_f16x8(o.l[1], lo);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = fmaf(f.f1, hi[j] + lo[j], v[j]);
    if constexpr (KIND == kMul) {
      if (!p.poly) {
        unpack_f16x8(o.r[0], hi);
        unpack_f16x8(o.r[1], lo);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(f.f2, hi[j] + lo[j], v[j]);
      }
    }
  }
  if (KIND == kLast) return 0.f;
  float s = 0.f, with[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) with[j] = v[j];
  if constexpr (KIND == kMul)
    if (p.with) unpack_f16x8(p.with == 1 ? o.l[0] : p.with == 2 ? o.r[0] : o.partner, with);   // (the hi part: a shift needs no more)
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fmaf(v[j], with[j], s);
  return s;
}

// The scalars' way through a launch.  Before the products: partial sums and means to registers; behind them (all waves): the factors.
template <int KIND, int NT>
struct OrthScalars {
  float part = 0.f, left = 0.f, right = 0.f;
  __device__ __forceinline__ void begin(const OrthProduct& p, int64_t skip4) {   // (nothing waits here)
    if ((KIND == kMul || (KIND == kGram && !p.first)) && (int)threadIdx.x < p.n_sums) part = p.sums_in[skip4 + threadIdx.x];
    if (KIND != kGram) left = p.means[skip4 + p.mean_left];
    if (KIND == kMul) right = p.means[skip4 + p.mean_right];
  }
  __device__ __forceinline__ OrthFactors end(const OrthProduct& p, int64_t skip4, int tile, float* shared) {   // shared: NT / 64 floats
    float s = 0.f;
    if (KIND < kUpdate) {
      if (KIND == kMul || !p.first)
        for (int i = threadIdx.x + NT; i < p.n_sums; i += NT) part += p.sums_in[skip4 + i];
      const float w = wave_sum(part);
      if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = w;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NT / 64; ++i) s += shared[i];
    }
    const OrthFactors f = orth_factors<KIND>(p, s, left, right);
    if (KIND < kUpdate && tile == 0 && threadIdx.x == 0) p.means[skip4 + p.mean_out] = f.mean;
    return f;
  }
};

template <int KIND, int BM, int BN, int WM, int WN, bool PLANES>
__global__ __launch_bounds__(512) void orth_phased_kernel(OrthProduct p, typename EndsOf<KIND>::type e) {
  constexpr int MI = WM / 32, NI = WN / 32, WAVES_N = BN / WN, CPR = WN / 4, LPR = WN / 8, NIT = 32 * LPR / 64;
  extern __shared__ uint4 smem[];
  __shared__ float shared[16];
  const OrthPlace at = orth_place<KIND, BM, BN>(p);
  const int64_t skip = at.matrix * p.matrix / 2, skip4 = at.matrix * p.matrix / 4;   // 2- and 4-byte elements
  p.A += skip;
  p.B += skip;
  OrthScalars<KIND, 512> scalars;
  scalars.begin(p, skip4);
  const int m0 = at.bm * BM, n0 = at.bn * BN;
  f32x16 acc[MI][NI];
  phased_products<MulF16, BM, BN, WM, WN, false, (KIND < kUpdate), PLANES>(acc, p, m0, n0, smem, [](int, int, int, uint32_t) {});
  const OrthFactors f = scalars.end(p, skip4, at.tile, shared);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave / WAVES_N, wn = wave % WAVES_N;
  // every wave's own: a strip of 32 rows in fp32 (16-byte chunks swizzled with the row), and its transpose in two planes of fp16
  constexpr int kStrip = 32 * CPR, kTurned = WN * 4;   // uint4
  uint4* own = smem + wave * (kStrip + 2 * kTurned);
  float4* strip = reinterpret_cast<float4*>(own);
  uint16_t* turned = reinterpret_cast<uint16_t*>(own + kStrip);
  const int r = lane & 31, khalf = lane >> 5, col_base = n0 + wn * WN;
  bool mirror = KIND < kUpdate && !in_lower_tile<BM, BN>(n0, m0 + BM - 1);   // some entry's image is not computed
  if constexpr (KIND == kLast) mirror = e.tall;                              // X leaves transposed
  bf16_t* out = p.out + skip;
  float sum = 0.f;
  // (X's entries are asked for one strip ahead; the m x m operands', of which there are more, at the strip's begin)
  constexpr int kAhead = KIND == kUpdate ? 2 : 1;
  OrthOld<KIND> old[kAhead][NIT];
  auto ask = [&](int mi) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      const int L = it * 64 + lane, row = m0 + wm * WM + mi * 32 + L / LPR, col = col_base + L % LPR * 8;
      if (row < p.M && col < p.N) {
        orth_ask<KIND>(p, skip, row, col, old[mi % kAhead][it]);
        if constexpr (KIND == kLast)
          if (e.kind == kEndMuon && !e.tall && row < e.rows && col < e.cols)
            load8(e.w + at.matrix * e.in_stride + (int64_t)row * e.ld_in + col, old[mi % kAhead][it].w);
      }
    }
  };
  if (kAhead == 2) ask(0);
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    const int row_base = m0 + wm * WM + mi * 32;
    if (row_base >= p.M) break;   // wave-uniform; rows end at a multiple of 64
    if (kAhead == 1) ask(mi);
    else if (mi + 1 < MI) ask(mi + 1);
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        strip[r * CPR + ((ni * 8 + 2 * g + khalf) ^ (r & (CPR - 1)))] =
            make_float4(acc[mi][ni][4 * g], acc[mi][ni][4 * g + 1], acc[mi][ni][4 * g + 2], acc[mi][ni][4 * g + 3]);
    wave_lds_sync();
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      const int L = it * 64 + lane, rr = L / LPR, c8 = L % LPR, row = row_base + rr, col = col_base + c8 * 8;
      const float4 x = strip[rr * CPR + ((2 * c8) ^ (rr & (CPR - 1)))], y = strip[rr * CPR + ((2 * c8 + 1) ^ (rr & (CPR - 1)))];
      if (col < p.N) {
        float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        const float s = orth_finish<KIND>(p, f, row, col, old[mi % kAhead][it], v);
        if constexpr (KIND == kLast) {
          if (!e.tall) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= 1.f / kScaleX;
            if (row < e.rows && col < e.cols) orth_leave(e, at.matrix, row, col, v, old[mi % kAhead][it].w);
            continue;
          }
        }
        sum += KIND >= kUpdate || in_lower_tile<BM, BN>(col, row) ? s : 2.f * s;
        uint16_t h[2][8];
        split8(v, h[0], h[1]);
#pragma unroll
        for (int pl = 0; pl < 2; ++pl) {
          if (KIND != kLast) *reinterpret_cast<uint4*>(out + pl * p.out_plane + (int64_t)row * p.ldo + col) = pack_f16x8(h[pl]);
          if (mirror) {
#pragma unroll
            for (int j = 0; j < 8; ++j) turned[pl * kTurned * 8 + (c8 * 8 + j) * 32 + (((rr >> 3) ^ (c8 & 3)) << 3) + (rr & 7)] = h[pl][j];
          }
        }
      }
    }
    wave_lds_sync();
    if (mirror) {
#pragma unroll
      for (int it = 0; it < WN * 4 / 64; ++it) {
        const int L = it * 64 + lane, n = L >> 2, ch = L & 3, to_row = col_base + n, to_col = row_base + ch * 8;
        const uint16_t* from = turned + n * 32 + ((ch ^ ((n >> 3) & 3)) << 3);
        if constexpr (KIND == kLast) {
          if (to_row < e.rows && to_col < e.cols) {
            float x[8], lo[8], w[8];
            if (e.kind == kEndMuon) load8(e.w + at.matrix * e.in_stride + (int64_t)to_row * e.ld_in + to_col, w);
            load_f16x8(from, x);
            load_f16x8(from + kTurned * 8, lo);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (x[j] + lo[j]) * (1.f / kScaleX);
            orth_leave(e, at.matrix, to_row, to_col, x, w);
          }
        } else if (to_row < p.N && !in_lower_tile<BM, BN>(to_row, to_col)) {
#pragma unroll
          for (int pl = 0; pl < 2; ++pl)
            *reinterpret_cast<uint4*>(out + pl * p.out_plane + (int64_t)to_row * p.ldo + to_col) =
                *reinterpret_cast<const uint4*>(from + pl * kTurned * 8);
        }
      }
      wave_lds_sync();
    }
  }
  if (KIND == kLast) return;
  const float w = wave_sum(sum);
  if (lane == 0) shared[8 + wave] = w;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += shared[8 + i];
    p.sums_out[skip4 + at.tile] = s;
  }
}

// Few tiles: 64 x 64 of them, four waves that share the reduction range, K tiles of 32 in turn, each through a ring of LDS stages of its own
// (as gemm_bf16_split_kernel does it): four, or two where a tile has both planes.
constexpr int kSmall = 64, kSmallK = 32, kSmallWaves = 4;
template <int KIND, bool PLANES>
__global__ __launch_bounds__(kSmallWaves * 64) void orth_split_kernel(OrthProduct p, typename EndsOf<KIND>::type ends) {
  constexpr int BKA = PLANES ? 2 * kSmallK : kSmallK, KS = BKA / 16, NS = PLANES ? 2 : 4, AHEAD = PLANES ? 2 : 3, CHK = BKA / 8, NT = kSmallWaves * 64, kVecs = kSmall * kSmall / 8 / NT;
  constexpr int kStage = 2 * kSmall * CHK;   // uint4
  constexpr bool TB = KIND < kUpdate;
  extern __shared__ uint4 smem[];
  __shared__ float shared[8];
  const OrthPlace at = orth_place<KIND, kSmall, kSmall>(p);
  const int64_t skip = at.matrix * p.matrix / 2, skip4 = at.matrix * p.matrix / 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = at.bm * kSmall, n0 = at.bn * kSmall;
  AsyncLoader<kSmall, 1, BKA, true, kSmall, kSmall, PLANES> ld_a;
  AsyncLoader<kSmall, 1, BKA, TB, kSmall, kSmall, PLANES> ld_b;
  ld_a.init(p.A + skip + (int64_t)m0 * p.lda, p.lda, kSmall, 0, lane, 0, p.a_plane);
  ld_b.init(p.B + skip + (TB ? (int64_t)n0 * p.ldb : n0), p.ldb, kSmall, 0, lane, 0, p.b_plane);
  constexpr int IPA = decltype(ld_a)::IPW, NV = IPA + decltype(ld_b)::IPW;
  uint4* ring = smem + wave * (NS * kStage);
  const uint32_t lds_ring = __builtin_amdgcn_readfirstlane((uint32_t)reinterpret_cast<uintptr_t>(ring));
  const uint64_t a0 = uniform_address(ld_a.base_), b0 = uniform_address(ld_b.base_);
  const uint32_t a_step = ld_a.tile_step_bytes(), b_step = ld_b.tile_step_bytes();
  const int nk = p.seg_tiles, mine = nk > wave ? (nk - wave + kSmallWaves - 1) / kSmallWaves : 0;
  auto issue = [&](int i) __attribute__((always_inline)) {   // this wave's i-th tile, into stage i % NS; past the end nothing
    if (i >= mine) return;
    const uint32_t kt = (uint32_t)(wave + i * kSmallWaves), dst = lds_ring + (uint32_t)(i % NS * kStage) * 16u;
    const uint64_t a = a0 + (uint64_t)a_step * kt, b = b0 + (uint64_t)b_step * kt;
#pragma unroll
    for (int v = 0; v < IPA; ++v) ld_a.issue_one_untracked(v, a, dst);
#pragma unroll
    for (int v = 0; v < NV - IPA; ++v) ld_b.issue_one_untracked(v, b, dst + (uint32_t)(kSmall * CHK) * 16u);
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int mi = 0; mi < 2; ++mi)
#pragma unroll
    for (int ni = 0; ni < 2; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mi][ni][r] = 0.f;
  // in front of the tiles, older than which nothing is counted: what the epilogue needs
  OrthScalars<KIND, NT> scalars;
  scalars.begin(p, skip4);
  OrthOld<KIND> old[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int e = i * NT + tid;
    const int row = m0 + e / (kSmall / 8), col = n0 + e % (kSmall / 8) * 8;
    orth_ask<KIND>(p, skip, row, col, old[i]);
    if constexpr (KIND == kLast)
      if (ends.kind == kEndMuon && !ends.tall && row < ends.rows && col < ends.cols)
        load8(ends.w + at.matrix * ends.in_stride + (int64_t)row * ends.ld_in + col, old[i].w);
  }
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) issue(i);
  for (int i = 0; i < mine; ++i) {
    // tile i has landed once at most the loads of the AHEAD - 1 tiles behind it are outstanding
    if (i + AHEAD - 1 < mine) __builtin_amdgcn_s_waitcnt(vmcnt_imm((AHEAD - 1) * NV));
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    asm volatile("" ::: "memory");
    const uint4* stage = ring + i % NS * kStage;
    bf16x8 af[KS][2], bfr[KS][2];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        af[ks][q] = read_frag<kSmall, BKA, true>(stage, q * 32, ks, lane);
        bfr[ks][q] = read_frag<kSmall, BKA, TB>(stage + kSmall * CHK, q * 32, ks, lane);
      }
    // the stage has been read: the loads issued after this point may overwrite it
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (AHEAD == NS) issue(i + AHEAD);   // into the stage just read
#pragma unroll
    for (int q = 0; q < kTileProducts<KS, PLANES>; ++q)
#pragma unroll
      for (int mi = 0; mi < 2; ++mi)
#pragma unroll
        for (int ni = 0; ni < 2; ++ni) acc[mi][ni] = MulF16::run(bfr[b_of<KS, PLANES>(q)][ni], af[a_of<KS, PLANES>(q)][mi], acc[mi][ni]);
    if (AHEAD < NS) issue(i + AHEAD);   // into the stage read in the previous trip
  }
  const OrthFactors f = scalars.end(p, skip4, at.tile, shared);
  constexpr int LD = kSmall + 4;   // floats per row
  __syncthreads();                 // every wave is done with its ring
  float* part = reinterpret_cast<float*>(smem);
  uint16_t* turned = reinterpret_cast<uint16_t*>(part + kSmallWaves * kSmall * LD);   // [plane][64 columns][64 rows, 8 more]
#pragma unroll
  for (int mi = 0; mi < 2; ++mi)
#pragma unroll
    for (int ni = 0; ni < 2; ++ni)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(part + (wave * kSmall + mi * 32 + (lane & 31)) * LD + ni * 32 + 8 * q + 4 * (lane >> 5)) =
            make_float4(acc[mi][ni][4 * q], acc[mi][ni][4 * q + 1], acc[mi][ni][4 * q + 2], acc[mi][ni][4 * q + 3]);
  __syncthreads();
  bool mirror = KIND < kUpdate && at.bm != at.bn && !p.whole;
  if constexpr (KIND == kLast) mirror = ends.tall;
  bf16_t* out = p.out + skip;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int e = i * NT + tid, rr = e / (kSmall / 8), c = e % (kSmall / 8) * 8;
    float v[8] = {};
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) {
      const float4 lo = *reinterpret_cast<const float4*>(part + (w * kSmall + rr) * LD + c);
      const float4 hi = *reinterpret_cast<const float4*>(part + (w * kSmall + rr) * LD + c + 4);
      v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
      v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
    }
    sum += orth_finish<KIND>(p, f, m0 + rr, n0 + c, old[i], v);
    if constexpr (KIND == kLast) {
      if (!ends.tall) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= 1.f / kScaleX;
        if (m0 + rr < ends.rows && n0 + c < ends.cols) orth_leave(ends, at.matrix, m0 + rr, n0 + c, v, old[i].w);
        continue;
      }
    }
    uint16_t x[2][8];
    split8(v, x[0], x[1]);
#pragma unroll
    for (int pl = 0; pl < 2; ++pl) {
      if (KIND != kLast) *reinterpret_cast<uint4*>(out + pl * p.out_plane + (int64_t)(m0 + rr) * p.ldo + n0 + c) = pack_f16x8(x[pl]);
      if (mirror) {
#pragma unroll
        for (int j = 0; j < 8; ++j) turned[(pl * kSmall + c + j) * (kSmall + 8) + rr] = x[pl][j];
      }
    }
  }
  const float w = wave_sum(sum);
  if (lane == 0) shared[4 + wave] = w;
  __syncthreads();
  if (mirror) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int e = i * NT + tid, n = e / (kSmall / 8), r8 = e % (kSmall / 8) * 8;
      const uint16_t* from = turned + n * (kSmall + 8) + r8;
      if constexpr (KIND == kLast) {
        if (n0 + n < ends.rows && m0 + r8 < ends.cols) {
          float v[8], lo[8], w[8];
          if (ends.kind == kEndMuon) load8(ends.w + at.matrix * ends.in_stride + (int64_t)(n0 + n) * ends.ld_in + m0 + r8, w);
          load_f16x8(from, v);
          load_f16x8(from + kSmall * (kSmall + 8), lo);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (v[j] + lo[j]) * (1.f / kScaleX);
          orth_leave(ends, at.matrix, n0 + n, m0 + r8, v, w);
        }
      } else {
#pragma unroll
        for (int pl = 0; pl < 2; ++pl)
          *reinterpret_cast<uint4*>(out + pl * p.out_plane + (int64_t)(n0 + n) * p.ldo + m0 + r8) =
              *reinterpret_cast<const uint4*>(from + pl * kSmall * (kSmall + 8));
      }
    }
  }
  if (KIND == kLast) return;
  if (tid == 0) {
    const float s = (shared[4] + shared[5]) + (shared[6] + shared[7]);
    p.sums_out[skip4 + at.tile] = mirror ? 2.f * s : s;
  }
}

// ---------------------------------------------------------------------------- on the way in and out

template <typename T, bool MUON>
__device__ __forceinline__ void orth_load(const OrthEnds& e, int64_t at, float (&u)[8]) {
  if constexpr (MUON) {
    float m[8], g[8];
    load8(e.m + at, m);
    if (e.nesterov) {
      load8(e.G + at, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = e.beta * m[j] + e.omb * (g[j] * e.inv_micro);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = m[j];
    }
  } else load8(static_cast<const T*>(e.in) + at, u);
}

// The new momentum, and what is orthogonalised.
__device__ __forceinline__ void orth_momentum(const OrthEnds& e, int64_t at, float (&u)[8]) {
  float m[8], g[8];
  load8(e.m + at, m);
  load8(e.G + at, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = g[j] * e.inv_micro;
    m[j] = e.beta * m[j] + e.omb * gj;
    u[j] = e.nesterov ? e.beta * m[j] + e.omb * gj : m[j];
  }
  store8(e.m + at, m);
}

// Momentum (muon) and the sums of squares, in 64 bits: fp32 squares of a small gradient would be nothing.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void orth_square_kernel(OrthEnds e) {
  __shared__ double shared[4];
  const int matrix = blockIdx.y, per_row = e.cols / 8;
  const int64_t n = (int64_t)e.rows * per_row;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row, at = matrix * e.in_stride + r * e.ld_in + (i - r * per_row) * 8;
    float u[8];
    if constexpr (MUON) orth_momentum(e, at, u);
    else orth_load<T, false>(e, at, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (double)u[j] * (double)u[j];
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) e.squares[matrix * e.matrix / 8 + blockIdx.x] = (shared[0] + shared[1]) + (shared[2] + shared[3]);
}

// 64 x 64 elements of the caller's matrix per workgroup; a tall one passes through LDS transposed.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void orth_start_kernel(OrthEnds e) {
  __shared__ double shared[4];
  __shared__ float turned[64][65];
  // from the last elements to the first: those the sums were taken of last may still be in the memory-side cache
  const int matrix = gridDim.z - 1 - blockIdx.z, tid = threadIdx.x;
  double s = 0.0;
  for (int i = tid; i < e.n_squares; i += 256) s += e.squares[matrix * e.matrix / 8 + i];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if ((tid & 63) == 0) shared[tid >> 6] = s;
  __syncthreads();
  s = (shared[0] + shared[1]) + (shared[2] + shared[3]);
  const double factor = s == 0.0 ? 0.0 : (double)kScaleX / sqrt(s);   // a matrix of zeros stays one
  // (blocks cover the padding too)
  const int r0 = (gridDim.y - 1 - blockIdx.y) * 64, c0 = (gridDim.x - 1 - blockIdx.x) * 64;
  bf16_t* X = e.X + matrix * e.matrix / 2;
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int r = r0 + (it * 256 + tid) / 8, c = c0 + tid % 8 * 8;
    float u[8] = {};
    if (r < e.rows && c < e.cols) {
      orth_load<T, MUON>(e, matrix * e.in_stride + (int64_t)r * e.ld_in + c, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = (float)((double)u[j] * factor);
    }
    if (e.tall) {
#pragma unroll
      for (int j = 0; j < 8; ++j) turned[c - c0 + j][r - r0] = u[j];
    } else {
      uint16_t hi[8], lo[8];
      split8(u, hi, lo);
      bf16_t* x = X + (int64_t)r * e.ldx + c;
      *reinterpret_cast<uint4*>(x) = pack_f16x8(hi);
      *reinterpret_cast<uint4*>(x + e.plane) = pack_f16x8(lo);
    }
  }
  if (!e.tall) return;
  __syncthreads();
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int c = (it * 256 + tid) / 8, r = tid % 8 * 8;
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = turned[c][r + j];
    uint16_t hi[8], lo[8];
    split8(u, hi, lo);
    bf16_t* x = X + (int64_t)(c0 + c) * e.ldx + r0 + r;
    *reinterpret_cast<uint4*>(x) = pack_f16x8(hi);
    *reinterpret_cast<uint4*>(x + e.plane) = pack_f16x8(lo);
  }
}

// ---------------------------------------------------------------------------- small matrices

// Matrices that fit into a CU's LDS, X and A with both their planes: everything in one launch, one workgroup per matrix.  A launch of the
// products above takes 4 to 6 us whatever the size and there are 17 of them; here a product is two barriers and 1 to 3.3 us, of which (fp32,
// 128 x 128) half is the product, matrix instructions (1.3 us) and fragments out of LDS, and a quarter the conversions on the way back.  (The
// next fragments read in front of a product's instructions, in registers of their own: 58 instead of 55 us for that size.)  A product's mean is
// its trace.
struct OrthSmall { int steps; float inv_m; float coef[3 * kOrthMaxSteps]; };

__device__ __forceinline__ void orth_first(const OrthEnds& e, int64_t at, float (&u)[8]) {
  if (e.kind == kEndMuon) orth_momentum(e, at, u);
  else if (e.kind == kEndBf16) orth_load<bf16_t, false>(e, at, u);
  else orth_load<float, false>(e, at, u);
}

template <int MP, int NP, bool SPLIT>
struct OrthInLds {
  static constexpr int NW = MP * NP / 1024 < 8 ? MP * NP / 1024 : 8, NT = NW * 64;   // waves: of one 32 x 32 block of X or more
  static constexpr int kXBlocks = MP * NP / 1024 / NW, kABlocks = MP == 128 ? 2 : 1;  // a wave's, side by side
  static constexpr int kAWaves = MP * MP / 1024 / kABlocks;                           // waves that have blocks of m x m matrices, the first ones
  static constexpr int kParts = NW / kAWaves < (NP == 1024 ? 4 : 8) ? NW / kAWaves : (NP == 1024 ? 4 : 8);   // of A's reduction, for all waves to work on it
  static constexpr int kPlaneX = MP * NP / 8, kPlaneA = MP * MP / 8;                  // uint4
  // the parts' sums meet where A comes to lie, or (32 rows) behind it
  static constexpr int kSums = (kParts - 1) * kAWaves * kABlocks * 256;               // uint4
  static constexpr size_t kLds = (2 * kPlaneX + (MP == 32 ? 2 * kPlaneA + kSums : 2 * kPlaneA)) * sizeof(uint4);
  static_assert(MP == 32 || kSums <= 2 * kPlaneA, "room for the parts' sums");

  // Rows of C elements in 16-byte chunks, swizzled.
  template <int C> static __device__ __forceinline__ int place(int row, int chunk) { return row * (C / 8) + (chunk ^ swz<(C > 128 ? 128 : C) / 8>(row)); }
  template <int C> static __device__ __forceinline__ uint2* four(uint4* plane, int row, int col) {   // neighbours of a row
    return reinterpret_cast<uint2*>(plane + place<C>(row, col >> 3)) + ((col >> 2) & 1);
  }
  template <int C> static __device__ __forceinline__ bf16x8 along(const uint4* plane, int row0, int ks, int lane) {   // the reduction runs along the rows
    return __builtin_bit_cast(bf16x8, plane[place<C>(row0 + (lane & 31), ks * 2 + (lane >> 5))]);
  }
  template <int C> static __device__ __forceinline__ bf16x8 across(const uint4* plane, int col0, int ks, int lane) {   // down them (as read_frag)
    const int t = (lane & 15) >> 2, k = ks * 16 + (lane >> 5) * 8 + t, col = col0 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)four<C>(const_cast<uint4*>(plane), k, col));
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)four<C>(const_cast<uint4*>(plane), k + 4, col));
    typedef short v8i16 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, (v8i16)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // acc[j] = rows row0.. of L times rows (ACROSS: columns) 32 (col + j).. of R, over K from the `from`-th 16 on
  template <int BLOCKS, int K, int CL, int CR, bool ACROSS>
  static __device__ __forceinline__ void multiply(f32x16 (&acc)[BLOCKS], const uint4* L, int plane_l, const uint4* R, int plane_r, int row0, int col0, int lane,
                                                  int from = 0) {
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
    constexpr int kUnroll = K < 64 ? K / 16 : 4;
#pragma unroll kUnroll
    for (int i = 0; i < K / 16; ++i) {
      const int ks = from + i;
      const bf16x8 a = along<CL>(L, row0, ks, lane);
      bf16x8 al = a;
      if (SPLIT) al = along<CL>(L + plane_l, row0, ks, lane);
#pragma unroll
      for (int j = 0; j < BLOCKS; ++j) {
        const bf16x8 b = ACROSS ? across<CR>(R, col0 + 32 * j, ks, lane) : along<CR>(R, col0 + 32 * j, ks, lane);
        acc[j] = MulF16::run(b, a, acc[j]);
        if (SPLIT) {
          const bf16x8 bl = ACROSS ? across<CR>(R + plane_r, col0 + 32 * j, ks, lane) : along<CR>(R + plane_r, col0 + 32 * j, ks, lane);
          acc[j] = MulF16::run(bl, a, acc[j]);
          acc[j] = MulF16::run(b, al, acc[j]);
        }
      }
    }
  }
  // The sums of A's parts, one after the other, in the first kAWaves waves.
  static __device__ __forceinline__ void join(f32x16 (&acc)[kABlocks], float* sums, int lane, int wave) {
    if (kParts == 1) return;
    const int part = wave / kAWaves, owner = wave % kAWaves;
    auto at = [&](int p, int j, int r) __attribute__((always_inline)) { return sums + ((((p - 1) * kAWaves + owner) * kABlocks + j) * 16 + r) * 64 + lane; };
    if (part > 0 && part < kParts)
#pragma unroll
      for (int j = 0; j < kABlocks; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) *at(part, j, r) = acc[j][r];
    __syncthreads();
    if (part == 0)
#pragma unroll 1
      for (int p = 1; p < kParts; ++p)
#pragma unroll
        for (int j = 0; j < kABlocks; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[j][r] += *at(p, j, r);
  }
  // A lane's part of a diagonal block's diagonal: of 16 entries none, or one, number `has`; `place` in a plane (fp16 numbers).
  struct Diagonal { int has, place; bool there; };
  static __device__ __forceinline__ Diagonal diagonal(int row0, int lane, int m) {
    const int l = lane & 31, row = row0 + l;
    return {((l >> 2) & 1) == lane >> 5 ? l / 8 * 4 + (l & 3) : -1, place<MP>(row, row >> 3) * 8 + (row & 7), ((l >> 2) & 1) == lane >> 5 && row < m};
  }
  // The mean of an m x m product's diagonal, to every thread; own: the thread's entry of it.  A barrier: all have read the product's operands.
  static __device__ __forceinline__ float mean_of(const f32x16 (&acc)[kABlocks], const Diagonal& d, int row0, int col0, int lane, int wave, bool mine,
                                                  float inv_m, float* shared, float& own) {
    float s = 0.f;
    own = 0.f;
    if (mine)
#pragma unroll
      for (int j = 0; j < kABlocks; ++j)
        if (row0 == col0 + 32 * j) {   // uniform
          uint32_t v[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) v[r] = __float_as_uint(acc[j][r]);
#pragma unroll
          for (int n = 8; n > 0; n >>= 1) {
            uint32_t upper = d.has & n ? ~0u : 0u;
            asm("" : "+v"(upper));   // (a mask it is: the compiler makes branches of a choice among 16)
#pragma unroll
            for (int r = 0; r < n; ++r) v[r] = (v[r + n] & upper) | (v[r] & ~upper);
          }
          own = __uint_as_float(v[0]);
          s = wave_sum(d.has >= 0 ? own : 0.f);
        }
    if (lane == 0) shared[wave] = s;
    __syncthreads();
    s = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += shared[w];
    return s * inv_m;
  }
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  // f1 (what is there) + f3 acc, in place.  OLD: whether f1 counts; LOW: whether the remainder is needed.
  template <int BLOCKS, int C, bool OLD, bool LOW>
  static __device__ __forceinline__ void finish(const f32x16 (&acc)[BLOCKS], uint4* hi, uint4* lo, int row, int col0, int lane, float f1, float f3) {
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = col0 + 32 * j + 8 * g + 4 * (lane >> 5);
        f16x4 *ph = reinterpret_cast<f16x4*>(four<C>(hi, row, col)), *pl = reinterpret_cast<f16x4*>(four<C>(lo, row, col));
        f16x4 h, l;
        if (OLD) { h = *ph; l = *pl; }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v = acc[j][4 * g + i] * f3;
          if (OLD) v = __builtin_fmaf(f1, (float)h[i], __builtin_fmaf(f1, (float)l[i], v));   // (one instruction each, fp16 operands included)
          h[i] = (_Float16)v;
          l[i] = (_Float16)__builtin_fmaf((float)h[i], -1.f, v);
        }
        *ph = h;
        if (LOW) *pl = l;
      }
  }
  // The same for an m x m product, less f3 mean on the diagonal.
  template <bool OLD, bool LOW>
  static __device__ __forceinline__ void finish_less(const f32x16 (&acc)[kABlocks], const Diagonal& d, float own, float mean, uint4* hi, uint4* lo, int row0,
                                                     int col0, int lane, float f1, float f3) {
    _Float16 *ph = reinterpret_cast<_Float16*>(hi) + d.place, *pl = reinterpret_cast<_Float16*>(lo) + d.place;
    const bool here = d.there && row0 >= col0 && row0 < col0 + 32 * kABlocks;
    float v = (own - mean) * f3;
    if (OLD && here) v = fmaf(f1, (float)*ph + (float)*pl, v);
    finish<kABlocks, MP, OLD, LOW>(acc, hi, lo, row0 + (lane & 31), col0, lane, f1, f3);
    if (here) {
      const _Float16 h = (_Float16)v;
      *ph = h;
      if (LOW) *pl = (_Float16)(v - (float)h);
    }
  }
};

template <int MP, int NP, bool SPLIT>
__global__ __launch_bounds__((OrthInLds<MP, NP, SPLIT>::NT)) void orth_small_kernel(OrthEnds e, OrthSmall p) {
  using In = OrthInLds<MP, NP, SPLIT>;
  constexpr int kVecs = MP * NP / 8 / In::NT, NBX = NP / 32, NBA = MP / 32;
  extern __shared__ uint4 smem[];
  __shared__ double squares[In::NW];
  __shared__ float shared[In::NW];
  uint4 *X = smem, *Xl = X + In::kPlaneX, *A = Xl + In::kPlaneX, *Al = A + In::kPlaneA;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), matrix = blockIdx.x;
  const int per_row = e.cols / 8, vecs = e.rows * per_row, m = e.tall ? e.cols : e.rows;

  // in
  float u[kVecs][8];
  double s = 0.0;
#pragma unroll
  for (int it = 0; it < kVecs; ++it) {
    const int i = it * In::NT + tid, r = i / per_row;
#pragma unroll
    for (int j = 0; j < 8; ++j) u[it][j] = 0.f;
    if (i < vecs) orth_first(e, matrix * e.in_stride + (int64_t)r * e.ld_in + (i - r * per_row) * 8, u[it]);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (double)u[it][j] * (double)u[it][j];
    X[i] = Xl[i] = make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if (lane == 0) squares[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < In::NW; ++w) s += squares[w];
  const double factor = s == 0.0 ? 0.0 : (double)kScaleX / sqrt(s);   // a matrix of zeros stays one
#pragma unroll
  for (int it = 0; it < kVecs; ++it) {
    const int i = it * In::NT + tid, r = i / per_row, c = (i - r * per_row) * 8;
    if (i >= vecs) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) u[it][j] = (float)((double)u[it][j] * factor);
    uint16_t hi[8], lo[8];
    split8(u[it], hi, lo);
    if (!e.tall) {
      X[In::template place<NP>(r, c >> 3)] = pack_f16x8(hi);
      Xl[In::template place<NP>(r, c >> 3)] = pack_f16x8(lo);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = In::template place<NP>(c + j, r >> 3) * 8 + (r & 7);
        reinterpret_cast<uint16_t*>(X)[at] = hi[j];
        reinterpret_cast<uint16_t*>(Xl)[at] = lo[j];
      }
    }
  }
  __syncthreads();

  const bool mine = wave < In::kAWaves;
  const int ablock = wave % In::kAWaves * In::kABlocks, part = wave / In::kAWaves, xblock = wave * In::kXBlocks;
  const int arow0 = ablock / NBA * 32, acol0 = ablock % NBA * 32, xrow0 = xblock / NBX * 32, xcol0 = xblock % NBX * 32;
  const int xrow = xrow0 + (lane & 31);
  const typename In::Diagonal diag = In::diagonal(arow0, lane, m);
  for (int step = 0; step < p.steps; ++step) {
    const float a = p.coef[3 * step], b = p.coef[3 * step + 1], c = p.coef[3 * step + 2];
    f32x16 acc[In::kABlocks];
    // A = X X'
    if (part < In::kParts)
      In::template multiply<In::kABlocks, NP / In::kParts, NP, NP, false>(acc, X, In::kPlaneX, X, In::kPlaneX, arow0, acol0, lane, part * (NP / In::kParts / 16));
    In::join(acc, reinterpret_cast<float*>(MP == 32 ? Al + In::kPlaneA : A), lane, wave);
    float own, sum = In::mean_of(acc, diag, arow0, acol0, lane, wave, mine, p.inv_m, shared, own);
    if (mine) In::template finish_less<false, true>(acc, diag, own, sum, A, Al, arow0, acol0, lane, 0.f, kScaleA / (kScaleX * kScaleX));
    const float mean = sum * (1.f / (kScaleX * kScaleX));
    __syncthreads();
    // P = a + b A + c A^2, in A's place
    if (mine) In::template multiply<In::kABlocks, MP, MP, MP, false>(acc, A, In::kPlaneA, A, In::kPlaneA, arow0, acol0, lane);
    sum = In::mean_of(acc, diag, arow0, acol0, lane, wave, mine, p.inv_m, shared, own);
    if (mine)
      In::template finish_less<true, SPLIT>(acc, diag, own, sum, A, Al, arow0, acol0, lane, (b + 2.f * c * mean) * (kScaleP / kScaleA),
                                            c * (kScaleP / (kScaleA * kScaleA)));
    const float t = sum * (1.f / (kScaleA * kScaleA));
    __syncthreads();
    // X = mean_P X + P' X
    f32x16 x[In::kXBlocks];
    In::template multiply<In::kXBlocks, MP, MP, NP, true>(x, A, In::kPlaneA, X, In::kPlaneX, xrow0, xcol0, lane);
    __syncthreads();
    In::template finish<In::kXBlocks, NP, true, true>(x, X, Xl, xrow, xcol0, lane, a + b * mean + c * (mean * mean + t), 1.f / kScaleP);
    __syncthreads();
  }

  // out
#pragma unroll 1
  for (int i = tid; i < vecs; i += In::NT) {
    const int r = i / per_row, c = (i - r * per_row) * 8;
    float w[8], v[8], lo[8];
    if (e.kind == kEndMuon) load8(e.w + matrix * e.in_stride + (int64_t)r * e.ld_in + c, w);
    if (!e.tall) {
      unpack_f16x8(X[In::template place<NP>(r, c >> 3)], v);
      unpack_f16x8(Xl[In::template place<NP>(r, c >> 3)], lo);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = In::template place<NP>(c + j, r >> 3) * 8 + (r & 7);
        v[j] = f16_float(reinterpret_cast<const uint16_t*>(X)[at]);
        lo[j] = f16_float(reinterpret_cast<const uint16_t*>(Xl)[at]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (v[j] + lo[j]) * (1.f / kScaleX);
    orth_leave(e, matrix, r, c, v, w);
  }
}

// ---------------------------------------------------------------------------- host

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A matrix's part of the workspace, in bytes from its start.
struct OrthLayout {
  int m, n, mp, np;
  int64_t x_plane, m_plane;                                  // bytes
  int64_t x[2], mat[3], x_sums, m_sums[2], squares, means, size;
  int n_squares;
};
constexpr int kMaxSquares = 256;
OrthLayout orth_layout(int rows, int cols) {
  OrthLayout l;
  l.m = rows < cols ? rows : cols;
  l.n = rows < cols ? cols : rows;
  l.mp = (int)up(l.m, kPad); l.np = (int)up(l.n, kPad);
  l.x_plane = up((int64_t)l.mp * l.np * 2, 256);
  l.m_plane = up((int64_t)l.mp * l.mp * 2, 256);
  const int64_t tm = l.mp / kPad, tn = l.np / kPad;   // sums: of the smallest tiles at most
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t was = at; at += up(bytes, 256); return was; };
  for (int64_t& x : l.x) x = take(2 * l.x_plane);
  for (int64_t& x : l.mat) x = take(2 * l.m_plane);
  l.x_sums = take(tm * tn * 4);
  for (int64_t& x : l.m_sums) x = take(tm * tm * 4);
  l.squares = take(kMaxSquares * 8); l.means = take(3 * 4);
  l.size = at;
  const int64_t chunks = ((int64_t)rows * (cols / 8) + 2047) / 2048;   // 8 vectors a thread
  l.n_squares = (int)(chunks < 1 ? 1 : chunks > kMaxSquares ? kMaxSquares : chunks);
  return l;
}

bool orth_ok(const OrthDesc& d) {
  if ((d.dtype != kF32 && d.dtype != kBF16) || d.count < 1 || d.rows < 1 || d.cols < 8 || d.cols % 8 || d.steps < 1 || d.steps > kOrthMaxSteps)
    return false;
  if (d.rows > 65535 * kPad || d.cols > 65535 * kPad || d.count > 65535) return false;
  const int64_t mp = up(d.rows < d.cols ? d.rows : d.cols, kPad), np = up(d.rows < d.cols ? d.cols : d.rows, kPad);
  // (byte offsets of 31 bits in an operand, of two planes behind one another in fp32; the number of the smallest tiles)
  return (d.dtype == kF32 ? mp * np * 2 <= (1ll << 30) : mp * np * 2 < (1ll << 31)) && mp * np / (kPad * kPad) * d.count <= 0x7fffffff;
}

constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
const float* orth_coef(const OrthDesc& d, int step) { return d.coef ? d.coef + 3 * step : kQuintic; }

// Whether the first two steps may be taken together: the polynomials a + b l + c l^2 of both stay within 3.5 (the default's a is 3.4445) on the
// eigenvalues l that A can have there, [0, 1] and what becomes of them.  What A_0 is off by grows with the first one squared, and fp16 holds their
// product up to 64.
bool orth_mild(const OrthDesc& d) {
  double s = 1.0;   // X's largest singular value
  for (int i = 0; i < 2; ++i) {
    const float* k = orth_coef(d, i);
    const double a = k[0], b = k[1], c = k[2], top = s * s, turn = -b / (2.0 * c), root = std::sqrt(std::max(0.0, 9.0 * b * b - 20.0 * a * c));
    auto P = [&](double l) { return std::fabs(a + b * l + c * l * l); };
    double most = std::max(P(0.0), P(top)), next = s * P(top);
    if (turn > 0.0 && turn < top) most = std::max(most, P(turn));
    if (!(most <= 3.5)) return false;
    // s P(s^2) is largest at the end or where a + 3 b l + 5 c l^2 = 0 (c = 0: a + 3 b l)
    for (const double l : {(-3.0 * b + root) / (10.0 * c), (-3.0 * b - root) / (10.0 * c), -a / (3.0 * b)})
      if (l > 0.0 && l < top) next = std::max(next, std::sqrt(l) * P(l));
    s = next;
  }
  return true;
}

template <typename K>
hipError_t more_lds(K kernel, size_t lds, bool (&configured)[64]) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidValue;
  if (configured[dev]) return hipSuccess;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  configured[dev] = e == hipSuccess;
  return e;
}

template <int KIND>
int orth_tiles(int M, int N, int bm, int bn) {   // of a matrix
  const int tm = ceil_div(M, bm), tn = ceil_div(N, bn);
  if (KIND >= kUpdate) return tm * tn;
  int n = 0;
  for (int i = 0; i < tm; ++i) n += std::min(tn, (i * bm + bm - 1) / bn + 1);
  return n;
}

template <int KIND, int BM, int BN, int WM, int WN>
hipError_t launch_phased_orth(OrthProduct p, typename EndsOf<KIND>::type e, int count, hipStream_t s) {
  constexpr size_t stages = 2 * (BM + BN) * (kPhasedK / 8) * sizeof(uint4), strips = 8 * (32 * (WN / 4) + 2 * WN * 4) * sizeof(uint4);
  constexpr size_t lds = stages > strips ? stages : strips;
  static_assert(lds + 64 <= 160 * 1024, "LDS of a CU");
  static bool configured[2][64] = {};
  auto kernel = p.a_plane ? orth_phased_kernel<KIND, BM, BN, WM, WN, true> : orth_phased_kernel<KIND, BM, BN, WM, WN, false>;
  const hipError_t err = more_lds(kernel, lds, configured[p.a_plane != 0]);
  if (err != hipSuccess) return err;
  p.tiles_n = ceil_div(p.N, BN);
  p.tiles = orth_tiles<KIND>(p.M, p.N, BM, BN);
  if (p.a_plane) p.K *= 2;
  p.seg_tiles = p.K / kPhasedK;
  p.total = p.tiles * count;
  hipLaunchKernelGGL(kernel, dim3(p.total), dim3(512), lds, s, p, e);
  return hipGetLastError();
}

// Whether 64 x 64 tiles cover all of a symmetric result.  Mirroring takes a launch about 0.9 us; the tiles above the diagonal take the operands'
// traffic, 2 us per 1000 of K and 256 tiles (as the table below has it), and nothing else while there are CUs without one.  Five steps, us in
// all tiles | lower ones: bf16 223 x 912 106 | 113, 506 x 2248 171 | 181, two of 600 x 2400 184 | 195; fp32 223 x 912 156 | 167, 414 x 472
// 155 | 160.
template <int KIND>
bool orth_whole(int M, int N, int K, int count) {
  if (KIND >= kUpdate) return false;
  const int64_t all = (int64_t)(M / kSmall) * (N / kSmall) * count, lower = (int64_t)orth_tiles<KIND>(M, N, kSmall, kSmall) * count;
  return all <= gemm_compute_units() && (all - lower) * K < 100000;
}

template <int KIND>
hipError_t launch_split_orth(OrthProduct p, typename EndsOf<KIND>::type e, int count, hipStream_t s) {
  constexpr size_t lds = kSmallWaves * 4 * 2 * kSmall * (kSmallK / 8) * sizeof(uint4);
  static_assert(kSmallWaves * kSmall * (kSmall + 4) * 4 + 2 * kSmall * (kSmall + 8) * 2 <= lds, "partial sums and the turned tile fit in the rings");
  static bool configured[2][64] = {};
  auto kernel = p.a_plane ? orth_split_kernel<KIND, true> : orth_split_kernel<KIND, false>;
  const hipError_t err = more_lds(kernel, lds, configured[p.a_plane != 0]);
  if (err != hipSuccess) return err;
  p.tiles_n = p.N / kSmall;
  p.whole = orth_whole<KIND>(p.M, p.N, p.K * (p.a_plane ? 2 : 1), count);
  p.tiles = p.whole ? p.M / kSmall * p.tiles_n : orth_tiles<KIND>(p.M, p.N, kSmall, kSmall);
  p.seg_tiles = p.K / kSmallK;
  p.total = p.tiles * count;
  hipLaunchKernelGGL(kernel, dim3(p.total), dim3(kSmallWaves * 64), lds, s, p, e);
  return hipGetLastError();
}

// The tile shapes, and what a launch is taken to cost in microseconds with r tiles per CU, R = ceil(r) rounds of them and K in thousands:
//   fixed + round R + round_k K R + tile r + tile_k K r
// (as TileCost in gemm_bf16.hip).  Fitted to the launches of 74 sizes (64 to 8192 rows, 64 to 16384 columns, up to 12 matrices, K of 64 to
// 49152; two planes: 50 of them) with every shape forced: the choice takes 1.001 of the best shape's time (geometric mean), at worst 1.05.
// 4096 x 4096 results, K = 4096, one plane, us in 256x256 | 192x256 | 128x256 | 128x128 | 64x64 tiles: symmetric 83 | 84 | 111 | 102 | 229, whole 123 | 156 | 142 | 147 | 265;
// six of 1024 x 1024, symmetric, K = 4096: 76 | 64 | 48 | 39 | 74.
struct OrthTile { int bm, bn; float fixed, round, round_k, tile, tile_k; };
constexpr OrthTile kOrthTiles[2][3][5] = {   // one plane of every operand, two
    {
        {{256, 256, 0.f, 12.32f, 13.24f, 11.61f, 7.07f}, {192, 256, 0.f, 11.17f, 10.65f, 6.75f, 5.83f}, {128, 256, 0.f, 9.27f, 7.37f, 4.87f, 4.66f},
         {128, 128, 7.27f, 0.f, 5.35f, 2.08f, 2.59f}, {64, 64, 4.51f, 1.65f, 2.67f, 0.f, 2.21f}},
        {{256, 256, 0.f, 14.09f, 15.11f, 26.6f, 1.59f}, {192, 256, 0.f, 12.26f, 11.85f, 14.7f, 3.44f}, {128, 256, 0.f, 10.06f, 8.03f, 9.22f, 3.83f},
         {128, 128, 7.1f, 0.f, 5.88f, 5.44f, 1.82f}, {64, 64, 3.01f, 2.88f, 3.07f, 0.29f, 1.97f}},
        {{256, 256, 0.f, 11.85f, 12.72f, 6.68f, 10.35f}, {192, 256, 0.f, 10.31f, 11.08f, 3.22f, 7.64f}, {128, 256, 1.86f, 6.71f, 8.78f, 2.13f, 5.36f},
         {128, 128, 6.23f, 0.37f, 5.37f, 2.69f, 2.23f}, {64, 64, 2.71f, 1.84f, 2.64f, 0.81f, 0.65f}},
    },
    {
        {{256, 256, 0.f, 12.62f, 39.67f, 7.36f, 23.8f}, {192, 256, 0.f, 11.31f, 29.99f, 6.81f, 18.24f},
         {128, 256, 0.f, 8.96f, 21.39f, 4.16f, 13.71f}, {128, 128, 2.75f, 4.62f, 12.8f, 0.f, 10.64f},
         {64, 64, 4.29f, 1.35f, 6.4f, 0.24f, 4.24f}},
        {{256, 256, 13.62f, 0.f, 43.89f, 19.06f, 7.57f}, {192, 256, 11.57f, 0.f, 33.74f, 13.72f, 8.46f},
         {128, 256, 0.f, 9.1f, 23.92f, 8.84f, 7.46f}, {128, 128, 2.84f, 3.4f, 15.64f, 1.93f, 7.11f},
         {64, 64, 3.68f, 1.18f, 8.59f, 1.08f, 2.16f}},
        {{256, 256, 0.f, 11.53f, 38.62f, 4.14f, 25.95f}, {192, 256, 0.f, 9.94f, 31.52f, 1.15f, 19.61f},
         {128, 256, 1.96f, 6.68f, 20.9f, 0.f, 16.39f}, {128, 128, 5.77f, 0.19f, 12.9f, 0.89f, 8.23f},
         {64, 64, 2.88f, 1.83f, 5.63f, 1.02f, 1.94f}},
    },
};

struct OrthChoice { int shape; double cost; };
template <int KIND>
OrthChoice orth_tile(int M, int N, int K, int count, bool planes) {
  OrthChoice best{0, 0.0};
  for (int i = 0; i < 5; ++i) {
    const OrthTile& t = kOrthTiles[planes][KIND < kUpdate ? KIND : kUpdate][i];
    const int64_t tiles = (int64_t)count * orth_tiles<KIND>(M, N, t.bm, t.bn);
    const double R = ceil_div(tiles, (int64_t)gemm_compute_units()), r = (double)tiles / gemm_compute_units(), k = K * 1e-3;
    const double cost = t.fixed + t.round * R + t.round_k * k * R + t.tile * r + t.tile_k * k * r;
    if (i == 0 || cost < best.cost) best = {i, cost};
  }
  return best;
}

template <int KIND>
hipError_t launch_product(const OrthProduct& p, const typename EndsOf<KIND>::type& e, int count, int* tiles, hipStream_t s) {   // tiles: of a matrix, the number of sums left
  const int i = orth_tile<KIND>(p.M, p.N, p.K, count, p.a_plane != 0).shape;
  *tiles = orth_tiles<KIND>(p.M, p.N, kOrthTiles[0][KIND < kUpdate ? KIND : kUpdate][i].bm, kOrthTiles[0][KIND < kUpdate ? KIND : kUpdate][i].bn);
  if (i == 4 && orth_whole<KIND>(p.M, p.N, p.K * (p.a_plane ? 2 : 1), count)) *tiles = p.M / kSmall * (p.N / kSmall);
  switch (i) {
    case 0: return launch_phased_orth<KIND, 256, 256, 128, 64>(p, e, count, s);
    case 1: return launch_phased_orth<KIND, 192, 256, 96, 64>(p, e, count, s);
    case 2: return launch_phased_orth<KIND, 128, 256, 64, 64>(p, e, count, s);
    case 3: return launch_phased_orth<KIND, 128, 128, 64, 32>(p, e, count, s);
    default: return launch_split_orth<KIND>(p, e, count, s);
  }
}

// The launches of all steps.
struct OrthRun {
  const OrthDesc& d;
  const OrthLayout& l;
  const OrthEnds& ends;
  char* ws;
  hipStream_t stream;
  bool split;                     // fp32: three products
  int x = 0, x_sums = 0, m_sums = 0, at_sums = 0;   // X's buffer; numbers of sums (0: X has norm 1) and the buffer of the m x m ones
  OrthProduct base;

  OrthRun(const OrthDesc& d_, const OrthLayout& l_, const OrthEnds& e, char* ws_, hipStream_t s) : d(d_), l(l_), ends(e), ws(ws_), stream(s), split(d_.dtype == kF32), base{} {
    base.matrix = l.size; base.m = l.m; base.inv_m = 1.f / (float)l.m;
    base.means = reinterpret_cast<float*>(ws + l.means);
  }
  bf16_t* at(int64_t off) const { return reinterpret_cast<bf16_t*>(ws + off); }
  float* sums(int64_t off) const { return reinterpret_cast<float*>(ws + off); }
  uint32_t to_lo(int64_t plane) const { return split ? (uint32_t)plane : 0u; }

  // mat[0] = A of X
  hipError_t gram() {
    OrthProduct p = base;
    p.A = p.B = at(l.x[x]);
    p.M = p.N = l.mp; p.K = l.np; p.lda = p.ldb = l.np;
    p.a_plane = p.b_plane = to_lo(l.x_plane);
    p.out = at(l.mat[0]); p.ldo = l.mp; p.out_plane = l.m_plane / 2;
    p.scale_out = kScaleA; p.mean_out = 0;
    p.first = x_sums == 0;
    p.sums_in = sums(l.x_sums); p.n_sums = x_sums;
    p.sums_out = sums(l.m_sums[at_sums = 0]);
    return launch_product<kGram>(p, {}, d.count, &m_sums, stream);
  }
  // mat[out] = mat[left] mat[right] (coef: a + b L + c L^2 instead); the sums that the next product, of out with mat[partner], takes its mean
  // from (partner = out: with itself).
  hipError_t mul(int out, int left, int right, float sl, float sr, float so, int partner, const float* coef) {
    OrthProduct p = base;
    p.A = at(l.mat[left]); p.B = at(l.mat[right]);
    p.M = p.N = p.K = p.lda = p.ldb = p.ldo = l.mp;
    p.a_plane = p.b_plane = to_lo(l.m_plane);
    p.out = at(l.mat[out]); p.out_plane = p.old_plane = l.m_plane / 2;
    p.left = p.A; p.right = p.B; p.partner = at(l.mat[partner]);
    p.with = partner == out ? 0 : partner == left ? 1 : partner == right ? 2 : 3;
    p.mean_left = left; p.mean_right = right; p.mean_out = out;
    p.scale_left = sl; p.scale_right = sr; p.scale_out = so;
    if (coef) { p.poly = 1; p.a = coef[0]; p.b = coef[1]; p.c = coef[2]; }
    p.sums_in = sums(l.m_sums[at_sums]); p.n_sums = m_sums;
    p.sums_out = sums(l.m_sums[at_sums ^= 1]);
    return launch_product<kMul>(p, {}, d.count, &m_sums, stream);
  }
  // X = mat[by] X; the last time to where it leaves for
  hipError_t update(int by, float scale, bool last) {
    OrthProduct p = base;
    p.A = at(l.mat[by]); p.B = at(l.x[x]);
    p.M = l.mp; p.N = l.np; p.K = l.mp; p.lda = l.mp; p.ldb = l.np;
    p.a_plane = to_lo(l.m_plane); p.b_plane = to_lo(l.x_plane);
    p.left = p.B; p.old_plane = p.out_plane = l.x_plane / 2;
    x ^= 1;
    p.out = at(l.x[x]); p.ldo = l.np;
    p.mean_left = by; p.scale_left = scale;
    p.sums_out = sums(l.x_sums);
    if (last) return launch_product<kLast>(p, ends, d.count, &x_sums, stream);
    return launch_product<kUpdate>(p, {}, d.count, &x_sums, stream);
  }
  const float* coef(int step) const { return orth_coef(d, step); }
  hipError_t one(int step) {
    hipError_t e = gram();
    if (e == hipSuccess) e = mul(1, 0, 0, kScaleA, kScaleA, kScaleP, 1, coef(step));
    return e == hipSuccess ? update(1, kScaleP, step + 1 == d.steps) : e;
  }
  hipError_t two() {   // the first ones
    hipError_t e = gram();                                                                  // A_0
    if (e == hipSuccess) e = mul(1, 0, 0, kScaleA, kScaleA, kScaleP, 0, coef(0));           // P_1
    if (e == hipSuccess) e = mul(2, 0, 1, kScaleA, kScaleP, kScaleA, 1, nullptr);           // U = A_0 P_1
    if (e == hipSuccess) e = mul(0, 2, 1, kScaleA, kScaleP, kScaleA, 0, nullptr);           // A_1 = U P_1
    if (e == hipSuccess) e = mul(2, 0, 0, kScaleA, kScaleA, kScaleP, 1, coef(1));           // P_2
    if (e == hipSuccess) e = mul(0, 2, 1, kScaleP, kScaleP, kScaleP, 0, nullptr);           // Q = P_2 P_1
    return e == hipSuccess ? update(0, kScaleP, false) : e;
  }
  hipError_t all() {
    // The first two steps on one pass over X, where a pass costs more than the three m x m products, and the launch (about 2 us), that the pair has
    // in its place: 1024 x 1024 to 2048 x 2048 from n = 2 m on.
    const double passes = orth_tile<kGram>(l.mp, l.mp, l.np, d.count, split).cost + orth_tile<kUpdate>(l.mp, l.np, l.mp, d.count, split).cost;
    const bool cheaper = passes > 3.0 * orth_tile<kMul>(l.mp, l.mp, l.mp, d.count, split).cost + 2.0;
    const bool pair = cheaper && d.steps >= 4 && orth_mild(d);
    hipError_t e = pair ? two() : one(0);
    for (int i = pair ? 2 : 1; i < d.steps && e == hipSuccess; ++i) e = one(i);
    return e;
  }
};

template <int MP, int NP>
hipError_t launch_small_orth(const OrthDesc& d, const OrthEnds& e, const OrthSmall& p, hipStream_t s) {
  constexpr size_t lds = OrthInLds<MP, NP, true>::kLds;
  static_assert(lds + 128 <= 160 * 1024, "LDS of a CU");
  static bool configured[2][64] = {};
  const bool split = d.dtype == kF32;
  auto kernel = split ? orth_small_kernel<MP, NP, true> : orth_small_kernel<MP, NP, false>;
  const hipError_t err = more_lds(kernel, lds, configured[split]);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(kernel, dim3((unsigned)d.count), dim3(OrthInLds<MP, NP, true>::NT), lds, s, e, p);
  return hipGetLastError();
}

// Small matrices: all that fit.  One matrix, five steps, us in one launch | in one per product: fp32 32 x 64 17 | 78, 32 x 1024 49 | 123,
// 64 x 64 19 | 76, 64 x 512 56 | 103, 128 x 128 54 | 99; bf16 15 | 70, 43 | 88, 17 | 68, 47 | 83, 39 | 85.  1024 of them, fp32, 32 x 64 23 |
// 275, 32 x 1024 223 | 889, 64 x 512 286 | 626, 128 x 128 265 | 622.
template <typename T, bool MUON>
hipError_t orth_run(const OrthDesc& d, OrthEnds e, float* workspace, hipStream_t s) {
  const OrthLayout l = orth_layout(d.rows, d.cols);
  char* ws = reinterpret_cast<char*>(workspace);
  e.rows = d.rows; e.cols = d.cols; e.tall = d.rows > d.cols;
  e.X = reinterpret_cast<bf16_t*>(ws + l.x[0]); e.plane = l.x_plane / 2; e.matrix = l.size; e.ldx = l.np;
  e.squares = reinterpret_cast<double*>(ws + l.squares); e.n_squares = l.n_squares;
  if ((l.m <= 32 && l.np <= 1024) || (l.mp == 64 && l.np <= 512) || l.np == 128) {
    OrthSmall p;
    p.steps = d.steps; p.inv_m = 1.f / (float)l.m;
    for (int i = 0; i < 3 * d.steps; ++i) p.coef[i] = d.coef ? d.coef[i] : kQuintic[i % 3];
    const int np = l.np == 64 ? 64 : l.np == 128 ? 128 : l.np <= 256 ? 256 : l.np <= 512 ? 512 : 1024;
    switch ((l.m <= 32 ? 32 : l.mp) * 2048 + np) {
      case 32 * 2048 + 64: return launch_small_orth<32, 64>(d, e, p, s);
      case 32 * 2048 + 128: return launch_small_orth<32, 128>(d, e, p, s);
      case 32 * 2048 + 256: return launch_small_orth<32, 256>(d, e, p, s);
      case 32 * 2048 + 512: return launch_small_orth<32, 512>(d, e, p, s);
      case 32 * 2048 + 1024: return launch_small_orth<32, 1024>(d, e, p, s);
      case 64 * 2048 + 64: return launch_small_orth<64, 64>(d, e, p, s);
      case 64 * 2048 + 128: return launch_small_orth<64, 128>(d, e, p, s);
      case 64 * 2048 + 256: return launch_small_orth<64, 256>(d, e, p, s);
      case 64 * 2048 + 512: return launch_small_orth<64, 512>(d, e, p, s);
      default: return launch_small_orth<128, 128>(d, e, p, s);
    }
  }
  const dim3 blocks((unsigned)(up(d.cols, kPad) / kPad), (unsigned)(up(d.rows, kPad) / kPad), (unsigned)d.count);
  hipLaunchKernelGGL((orth_square_kernel<T, MUON>), dim3((unsigned)l.n_squares, (unsigned)d.count), dim3(256), 0, s, e);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((orth_start_kernel<T, MUON>), blocks, dim3(256), 0, s, e);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  return OrthRun(d, l, e, ws, s).all();
}

bool matrix_ok(const OrthDesc& d, int ld, int64_t stride) {
  return ld >= d.cols && ld % 8 == 0 && stride % 8 == 0 && (d.count == 1 || stride > 0) && ld <= (1 << 30);
}

// Whether no two of the matrices share an element: the distance of two is not within `cols` of a number of rows that both have.
bool apart(const OrthDesc& d, int ld, int64_t stride) {
  for (int64_t i = 1, at = stride; i < d.count && at < (int64_t)(d.rows - 1) * ld + d.cols; ++i, at += stride) {
    const int64_t row = at / ld, col = at % ld;
    if (col < d.cols || (ld - col < d.cols && row + 1 < d.rows)) return false;
  }
  return true;
}

}  // namespace

int64_t orthogonalize_workspace(const OrthDesc& d) {   // floats
  OrthDesc one = d;
  one.steps = 1;
  if (!orth_ok(one)) return 0;
  return orth_layout(d.rows, d.cols).size / 4 * d.count;
}

hipError_t orthogonalize(const OrthDesc& d, const void* in, int ld_in, int64_t in_stride, void* out, int ld_out, int64_t out_stride,
                         float* workspace, hipStream_t stream) {
  if (!orth_ok(d) || !matrix_ok(d, ld_in, in_stride) || !matrix_ok(d, ld_out, out_stride) || !in || !out || !workspace || !aligned16(in) ||
      !aligned16(out) || !aligned16(workspace) || !apart(d, ld_out, out_stride) ||
      (in == out && d.count > 1 && (ld_in != ld_out || in_stride != out_stride)))
    return hipErrorInvalidValue;
  OrthEnds e{};
  e.kind = d.dtype == kF32 ? kEndF32 : kEndBf16;
  e.in = in; e.out = out; e.ld_in = ld_in; e.ld_out = ld_out; e.in_stride = in_stride; e.out_stride = out_stride;
  return d.dtype == kF32 ? orth_run<float, false>(d, e, workspace, stream) : orth_run<bf16_t, false>(d, e, workspace, stream);
}

hipError_t muon_step(const OrthDesc& d, const MuonDesc& u, float* workspace, hipStream_t stream) {
  if (!orth_ok(d) || !matrix_ok(d, u.ld, u.stride) || !u.w_cur || !u.w_next || !u.m || !u.G || !workspace || !aligned16(u.w_cur) ||
      !aligned16(u.w_next) || !aligned16(u.m) || !aligned16(u.G) || !aligned16(u.w_next_lp) || !aligned16(workspace) || !apart(d, u.ld, u.stride))
    return hipErrorInvalidValue;
  OrthEnds e{};
  e.kind = kEndMuon;
  e.w = u.w_cur; e.G = u.G; e.w_next = u.w_next; e.m = u.m; e.w_lp = u.w_next_lp; e.ld_in = u.ld; e.in_stride = u.stride;
  e.beta = u.beta; e.omb = (float)(1.0 - (double)u.beta); e.nesterov = u.nesterov; e.inv_micro = u.inv_m;
  e.lr = (float)((double)u.lr * (double)u.scale); e.keep = (float)(1.0 - (double)u.lr * (double)u.decay);
  return orth_run<float, true>(d, e, workspace, stream);
}

}  // namespace k2bw
