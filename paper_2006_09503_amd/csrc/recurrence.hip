// Gated linear recurrence over packed gates [b*s, 3h] (columns F | C | R), per sequence and channel:
//   f = sigmoid(F), u = 1 - f = sigmoid(-F);  h_t = f_t h_(t-1) + u_t C_t;  o_t = h_t R_t sigmoid(R_t).
// Backward, from the last token to the first, with g_t what arrives at h_t:
//   g_t = dO_t R_t sigmoid(R_t) + B_(t+1),  B_t = f_t g_t;
//   dC_t = u_t g_t,  dF_t = g_t (h_(t-1) - C_t) f_t u_t,  dR_t = dO_t h_t sigmoid(R_t) (1 + R_t sigmoid(-R_t)).
// (u is computed from F by itself: 1 - f has no digits left where a memory is long.)
//
// Both directions are scans with maps x -> A x + H, in a single pass with look back (Merrill and Garland, 2016); the maps compose: (A1, H1) then (A2, H2) is (A1 A2, A2 H1 + H2).  A workgroup owns a
// tile of rows x 128 channels (bf16; 64 in fp32: 256 bytes of a row).  A sub -- a wave, or half of one in fp32 -- holds 8 consecutive rows of
// it, two channels per lane, in registers, and reduces them to their map; the subs' maps meet in LDS, the tile's own map is published, the
// state that enters the tile comes from the tiles in front of it (behind it, backward), and the rows are gone through once more, from
// registers.  So every gate is read from HBM once and every output written once, however long the sequence and however few the channels.
//
// Between tiles: the maps of tiles and of blocks of 8 tiles are 8-byte words, the states at the blocks' ends 4-byte words, each written and
// read by relaxed atomics at device scope and each its own flag: all bits set means "not there yet" (a NaN of that pattern is replaced by
// another NaN), so no fence and no order between two words is needed.  A tile asks for the maps of its block's tiles in front of it, which
// depend on nothing, and for the state at the end of the block before: the subs look at as many blocks at once, so a finished state moves
// on by 64 tiles in a round of loads (with tiles alone, 8 at a time: 160 instead of 102 us for 32768 x 1024 bf16, forward).
// The tiles of a chain (a group of channels of a sequence) are numbered by a ticket that a workgroup draws when it starts: a workgroup
// waits only for workgroups of its chain that have started, and of those that wait the one with the lowest ticket waits for nobody, so
// every wait ends.
//
// fp32: bound by its streams (32768 x 1000: forward 139 us, backward 207, where the same rows loaded and stored with nothing computed take 124 and 215;
// rows of 4000 bytes share lines).  bf16: 34 and 60 us for 2048 x 8192, where the streams alone take 21 and 37: vector instructions are at work half of
// the time and waves wait half of theirs (profiles/operators_counters.txt), the latencies of a workgroup's life (ticket, loads, maps, stores).  The
// launches that clear the words and finish the sums come on top.  Two workgroups of eight waves on a CU: forward 94 registers, backward 128, which is all there are for
// two.  Forced to more, the spills cost more than the waves bring (forward at 80 registers 55 us, backward at 96 144); 16 waves: even
// forward, 8 % behind backward; 4 rows per sub: 10 % behind.
//
// The forward keeps the state in front of every 64th row (fp32); the backward rebuilds the states in between from it.
#include "kernels.hpp"

namespace k2bw {
namespace {

constexpr int kRecSave = 64;        // rows between two kept states
constexpr int kRecWaves = 8, kRecMaxThreads = 64 * kRecWaves;
constexpr int kRecBlock = 8;        // tiles of a block, at most the subs of a workgroup where there is more than one tile
constexpr int kRecTicket = 16;      // words from one ticket to the next: lines of their own, or the draws queue up (4096 of one: 20 us)

// Lanes side by side in a row, two channels each: 256 bytes of it (rows of 128 bytes: 51 instead of 44 us for the backward pass's seven
// streams of 2048 x 8192 bf16, with nothing computed).
template <typename T> constexpr int kRecLanes = sizeof(T) == 2 ? 64 : 32;

template <typename T> struct Pair;   // two neighbouring channels
template <> struct Pair<float> {
  typedef uint32_t type __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float2 floats(type v) { return make_float2(__uint_as_float(v.x), __uint_as_float(v.y)); }
  static __device__ __forceinline__ type pack(float a, float b) { return type{__float_as_uint(a), __float_as_uint(b)}; }
  static __device__ __forceinline__ type infinities() { return type{0x7f800000u, 0x7f800000u}; }
  static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t lane, uint32_t row) { return __builtin_amdgcn_raw_buffer_load_b64(r, lane, row, 0); }
  static __device__ __forceinline__ void store(type v, __amdgpu_buffer_rsrc_t r, uint32_t lane, uint32_t row) { __builtin_amdgcn_raw_buffer_store_b64(v, r, lane, row, 0); }
  // 2^t with what the product t = -x log2(e) and that constant lose put back
  static __device__ __forceinline__ float exp_neg(float x) {
    const float y = __builtin_amdgcn_fmed3f(x, -200.f, 200.f);
    const float lost = fmaf(-1.92596303e-8f, y, fmaf(-1.44269502162933350f, y, 1.44269502162933350f * y));
    const float z = __builtin_elementwise_minimum(__builtin_amdgcn_exp2f(-1.44269502162933350f * x), 0x1p124f);   // (an infinity times nothing lost)
    return fmaf(z * 0.69314718f, lost, z);
  }
};
template <> struct Pair<bf16_t> {
  using type = uint32_t;
  static __device__ __forceinline__ type infinities() { return 0x7f807f80u; }
  static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t lane, uint32_t row) { return __builtin_amdgcn_raw_buffer_load_b32(r, lane, row, 0); }
  static __device__ __forceinline__ void store(type v, __amdgpu_buffer_rsrc_t r, uint32_t lane, uint32_t row) { __builtin_amdgcn_raw_buffer_store_b32(v, r, lane, row, 0); }
  static __device__ __forceinline__ float2 floats(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
  // (off by x 2^-24 of the value: far under the step of a bf16 result, and like a few more roundings in what leaves as fp32)
  static __device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(-1.44269504088896341f * x); }
};

// sigmoid(x) = 1 / (1 + z) and sigmoid(-x) = z / (1 + z), z = exp(-x), both to full relative precision.  z ends at 2^124, where the one
// is 2^-124 and the other 1 (a reciprocal further down would be flushed to zero); a NaN stays one.  The reciprocal instruction's own error
// goes the same way at every token, and a memory of hundreds adds it up.  fp32: near 1 the one is 1 minus the other, off by the rounding of
// that alone (32768 tokens: results off by 2.2e-7 instead of 8.7e-7).  bf16, whose states and their gradients leave in fp32: a Newton step, an
// instruction less (the carried gradient off by 3.6e-7 instead of 1.2e-6; backward of 2048 x 8192 59 us without it, 60 with, 63 the other way).
template <typename T>
__device__ __forceinline__ void sigmoids(float x, float& pos, float& neg) {
  const float z = __builtin_elementwise_minimum(Pair<T>::exp_neg(x), 0x1p124f);
  const float d = 1.0f + z;
  pos = __builtin_amdgcn_rcpf(d);
  if (sizeof(T) == 2) pos = fmaf(fmaf(-d, pos, 1.0f), pos, pos);
  neg = z * pos;
  if (sizeof(T) == 4) pos = z <= 1.0f ? 1.0f - neg : pos;
}
// R sigmoid(R) and its slope sigmoid(R) (1 + R sigmoid(-R)).  Below -85 both are under 1e-34, and R counts as -85: a gate of the type's lowest
// value is closed, and no exponential overflows.
template <typename T>
__device__ __forceinline__ float gate_of(float R) {
  const float x = __builtin_elementwise_maximum(R, -85.f);
  return x * __builtin_amdgcn_rcpf(1.0f + Pair<T>::exp_neg(x));
}
template <typename T>
__device__ __forceinline__ float gate_of(float R, float& slope) {
  const float x = __builtin_elementwise_maximum(R, -85.f), s = __builtin_amdgcn_rcpf(1.0f + Pair<T>::exp_neg(x)), v = x * s;
  slope = fmaf(v, 1.f - s, s);
  return v;
}

// The value is computed here: left alone, the compiler puts the second half of a sigmoid off to where the result is used, and keeps what
// that takes, twice the registers, alive over the scan (128 registers and 56 spilled instead of under 128).
__device__ __forceinline__ void here(float (&v)[2]) { asm volatile("" : "+v"(v[0]), "+v"(v[1])); }
// The same number, for all the compiler knows another one: rows' masked offsets are made again (two instructions) where they are used next,
// and not kept in a register each from the loads to the last stores.
__device__ __forceinline__ int again(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

struct RecParams {
  const void* gates; const void* d_o; void* out;   // forward: out = o; backward: out = dgates
  const int32_t* lens;
  const float* carry_in; float* carry_out;         // state (forward), its gradient (backward): [b, h] or null
  float* saved;
  uint64_t *maps, *block_maps; uint32_t* block_ends;   // [tiles or blocks][b][h]
  uint32_t* tickets;                               // [chains][kRecTicket]
  float* sums;                                     // backward: [b * tiles][3h] column sums, or null
  int b, s, h, tiles, groups, rows;                // rows: of a tile
  uint32_t near;                                   // neighbouring groups on one XCD (whose workgroups are every eighth)
};

__device__ __forceinline__ uint32_t word_of(float v) {   // never the pattern that means "not there"
  return v != v ? 0x7fc00000u : __float_as_uint(v);
}
__device__ __forceinline__ void put_map(uint64_t* p, float A, float H) {
  __hip_atomic_store(p, ((uint64_t)word_of(H) << 32) | word_of(A), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put_end(uint32_t* p, float v) {
  __hip_atomic_store(p, word_of(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// `n` words of "not there yet" (in fours) behind `tickets` ones.
__global__ __launch_bounds__(256) void recurrence_clear_kernel(uint4* p, int64_t tickets, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t v = i < tickets ? 0u : ~0u;
  if (i < tickets + n) p[i] = make_uint4(v, v, v, v);
}

// The tile and its place.  Workgroups are dealt to the chains (one group of channels of one sequence) in turn; `turn` is the chain's ticket.
// (Starting on the tile that the workgroup's number stands for, and looking at the ticket later, gained 1 us in 40 where that number was
// right, and lost up to 40 in 140 where it was not.)
struct RecPlace { int turn, n, c0, row0, sub, lane, nsub, len; bool active; };
template <int W>
__device__ __forceinline__ RecPlace place_of(const RecParams& p, uint32_t* shared_ticket, bool backward, int L) {
  const uint32_t chains = (uint32_t)p.groups * p.b, span = 8 * p.near, in = blockIdx.x % span;
  const uint32_t id = blockIdx.x < gridDim.x / span * span ? blockIdx.x - in + in % 8 * p.near + in / 8 : blockIdx.x;
  const uint32_t chain = id % chains;
  RecPlace q;
  q.turn = 0;
  q.n = chain / p.groups;
  q.len = p.lens ? min(max(p.lens[q.n], 0), p.s) : p.s;   // (on its way with the ticket)
  if (p.tiles > 1) {
    if (threadIdx.x == 0) *shared_ticket = atomicAdd(p.tickets + (int64_t)chain * kRecTicket, 1u);
    __syncthreads();
    q.turn = __builtin_amdgcn_readfirstlane((int)*shared_ticket);
  }
  q.lane = threadIdx.x % W; q.sub = threadIdx.x / W; q.nsub = blockDim.x / W;
  q.c0 = ((chain - q.n * p.groups) * W + q.lane) * 2;
  q.active = q.c0 < p.h;
  q.row0 = (backward ? p.tiles - 1 - q.turn : q.turn) * p.rows + q.sub * L;
  return q;
}

__device__ __forceinline__ float4 unpack_maps(uint64_t m0, uint64_t m1) {
  return make_float4(__uint_as_float((uint32_t)m0), __uint_as_float((uint32_t)(m0 >> 32)), __uint_as_float((uint32_t)m1), __uint_as_float((uint32_t)(m1 >> 32)));
}
__device__ __forceinline__ uint64_t peek(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t peek(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float2 through(const float4& m, float2 x) { return make_float2(fmaf(m.x, x.x, m.y), fmaf(m.z, x.y, m.w)); }
__device__ __forceinline__ float4 then(const float4& first, const float4& second) {
  return make_float4(first.x * second.x, fmaf(second.x, first.y, second.y), first.z * second.z, fmaf(second.z, first.w, second.w));
}

// The caller's state, to LDS, by the tiles that start from it; in front of the barrier that their own maps are published behind.  The last
// tile waits for all maps, so nobody is left to read the state when it stores the new one, which may go to the same place.
template <int W>
__device__ __forceinline__ void take_carry(const RecParams& p, const RecPlace& q, float4 (*win)[W]) {
  if (p.carry_in && q.turn < kRecBlock && q.sub == 0 && q.active) {
    const float2 v = *reinterpret_cast<const float2*>(p.carry_in + (int64_t)q.n * p.h + q.c0);
    win[0][q.lane] = make_float4(v.x, v.y, 0.f, 0.f);
  }
}

// The state that enters this tile, of a thread's two channels, in one order of operations whatever had got how far: the state that enters the
// tile's block, through the maps of the block's tiles in front of this one.  The former is the nearest finished one, through the maps of
// the blocks in between, one after the other, which is what those blocks do themselves.
// own: this tile's map, of the threads of sub `teller`, which publishes the block's.
template <int W>
__device__ __forceinline__ float2 look_back(const RecParams& p, const RecPlace& q, const float4& own, int teller, float4 (*near)[W], float4 (*win)[W]) {
  const int64_t step = (int64_t)p.b * p.h, col = (int64_t)q.n * p.h + q.c0;
  const int block = q.turn / kRecBlock, pos = q.turn % kRecBlock;
  if (q.sub < pos && q.active) {   // the block's tiles in front: sub j asks for tile j
    const uint64_t* m = p.maps + (int64_t)(block * kRecBlock + q.sub) * step + col;
    uint64_t m0, m1;
    while ((m0 = peek(m)) == ~0ull || (m1 = peek(m + 1)) == ~0ull) __builtin_amdgcn_s_sleep(1);
    near[q.sub][q.lane] = unpack_maps(m0, m1);
  }
  __syncthreads();
  const bool tell = pos == kRecBlock - 1 && q.sub == teller && q.active;
  float4 whole = make_float4(1.f, 0.f, 1.f, 0.f);
  if (tell) {
#pragma unroll 2
    for (int j = 0; j < pos; ++j) whole = then(whole, near[j][q.lane]);
    whole = then(whole, own);
    put_map(p.block_maps + block * step + col, whole.x, whole.y);
    put_map(p.block_maps + block * step + col + 1, whole.z, whole.w);
  }
  float2 in = make_float2(0.f, 0.f);
  if (block == 0) {
    if (p.carry_in && q.active) in = make_float2(win[0][q.lane].x, win[0][q.lane].y);   // (see take_carry)
  } else {
    const int t = block - 1 - q.sub, count = min(block, q.nsub);
    const bool look = t >= 0 && q.active;
    const uint64_t* m = p.block_maps + (look ? t * step + col : 0);
    const uint32_t* e = p.block_ends + (look ? t * step + col : 0);
    bool finished = false;   // the block that this sub looks at
    for (;;) {
      while (look && !finished) {
        const uint32_t e0 = peek(e), e1 = peek(e + 1);
        const uint64_t m0 = peek(m), m1 = peek(m + 1);
        finished = e0 != ~0u && e1 != ~0u;
        if (finished) win[q.sub][q.lane] = make_float4(-1.f, __uint_as_float(e0), -1.f, __uint_as_float(e1));   // a factor no map has
        else if (m0 != ~0ull && m1 != ~0ull) win[q.sub][q.lane] = unpack_maps(m0, m1);
        else {
          __builtin_amdgcn_s_sleep(1);
          continue;
        }
        break;
      }
      __syncthreads();
      int j = 0;
      if (q.active) {
#pragma unroll 1
        while (j < count && win[j][q.lane].x != -1.f) ++j;
      }
      if (!__syncthreads_and(j < count)) continue;
      if (q.active) {
        in = make_float2(win[j][q.lane].y, win[j][q.lane].w);
#pragma unroll 2
        while (--j >= 0) in = through(win[j][q.lane], in);
      }
      break;
    }
  }
  if (tell) {
    const float2 end = through(whole, in);
    put_end(p.block_ends + block * step + col, end.x);
    put_end(p.block_ends + block * step + col + 1, end.y);
  }
#pragma unroll 2
  for (int j = 0; j < pos; ++j) in = through(near[j][q.lane], in);
  return in;
}

// The rows of a wave in a matrix of rows `ld` elements apart, through buffer accesses: the wave's base and the row's offset are scalars, the
// lane's 32-bit offset serves all rows, and a lane that has no business in a row has an offset past the buffer's end: it reads zero and
// writes nothing.
template <typename T>
struct RecRows {
  using Raw = typename Pair<T>::type;
  static constexpr uint32_t kNowhere = 0x80000000u;
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t lane, ld;
  __device__ __forceinline__ RecRows(const void* p, int64_t ld_, const RecPlace& q, int s, int L) : ld((uint32_t)ld_ * (uint32_t)sizeof(T)) {
    const int64_t first = (int64_t)q.n * s + __builtin_amdgcn_readfirstlane(q.row0);
    T* base = static_cast<T*>(const_cast<void*>(p)) + first * ld_ + __builtin_amdgcn_readfirstlane(q.c0);
    rsrc = __builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7fffffff, 0x00020000);
    lane = ((kRecLanes<T> == 32 && (threadIdx.x & 32)) ? (uint32_t)L * ld : 0u) + (uint32_t)(q.lane * 2 * sizeof(T));
  }
  __device__ __forceinline__ Raw load(int i, uint32_t off, bool there) const {   // off: bytes in the row, uniform
    return Pair<T>::load(rsrc, there ? lane : kNowhere, (uint32_t)i * ld + off);
  }
  __device__ __forceinline__ void store(Raw v, int i, uint32_t off, bool there) const {
    Pair<T>::store(v, rsrc, there ? lane : kNowhere, (uint32_t)i * ld + off);
  }
  // Rows behind the last token up to the sequence's end: zeros, whatever the state (what the loops compute there is zero times it).
  __device__ __forceinline__ void zeros(int from, int to, uint32_t off) const {
    for (int i = max(from, 0); i < to; ++i) Pair<T>::store(Pair<T>::pack(0.f, 0.f), rsrc, lane + (uint32_t)i * ld, off);
  }
};

template <typename T, int L>
__global__ __launch_bounds__(kRecMaxThreads) void recurrence_fwd_kernel(RecParams p) {
  using P = Pair<T>;
  using Raw = typename P::type;
  constexpr int W = kRecLanes<T>, S = kRecMaxThreads / W;
  __shared__ float4 maps[S][W], win[S][W], near[kRecBlock][W];
  __shared__ uint32_t ticket;
  const RecPlace q = place_of<W>(p, &ticket, false, L);
  const uint32_t gate = (uint32_t)p.h * (uint32_t)sizeof(T);   // bytes from F to C, from C to R
  const int lim = q.active ? min(q.len - q.row0, L) : 0;       // rows of this sub that are real
  float f[L][2], x[L][2], r[L][2];                             // f, u C, R sigmoid(R)
  float4 own = make_float4(1.f, 0.f, 1.f, 0.f);                // A, H of either channel
  {
    const RecRows<T> src(p.gates, 3 * (int64_t)p.h, q, p.s, L);
    Raw F[L], C[L], R[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool real = i < lim;
      F[i] = src.load(i, 0, real);
      C[i] = src.load(i, gate, real);
      R[i] = src.load(i, 2 * gate, real);
    }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const float2 F2 = P::floats(i < lim ? F[i] : P::infinities()), C2 = P::floats(C[i]), R2 = P::floats(R[i]);   // past the end: f = 1, u = 0
      float u0, u1;
      sigmoids<T>(F2.x, f[i][0], u0);
      sigmoids<T>(F2.y, f[i][1], u1);
      x[i][0] = u0 * C2.x;
      x[i][1] = u1 * C2.y;
      r[i][0] = gate_of<T>(R2.x);
      r[i][1] = gate_of<T>(R2.y);
      here(f[i]);
      here(x[i]);
      here(r[i]);
      own.y = fmaf(f[i][0], own.y, x[i][0]);
      own.w = fmaf(f[i][1], own.w, x[i][1]);
      own.x *= f[i][0];
      own.z *= f[i][1];
    }
  }
  maps[q.sub][q.lane] = own;
  take_carry<W>(p, q, win);
  __syncthreads();
  float4 pre = make_float4(1.f, 0.f, 1.f, 0.f);   // of the subs in front
#pragma unroll 2
  for (int j = 0; j < q.sub; ++j) {
    pre = then(pre, maps[j][q.lane]);
  }
  const bool last_sub = q.sub == q.nsub - 1 && q.active;
  const int64_t at = (int64_t)q.n * p.h + q.c0, word = (int64_t)q.turn * p.b * p.h + at;
  const float4 all = then(pre, own);
  if (p.tiles > 1 && last_sub) {
    put_map(p.maps + word, all.x, all.y);
    put_map(p.maps + word + 1, all.z, all.w);
  }
  const float2 in = look_back<W>(p, q, all, q.nsub - 1, near, win);
  if (last_sub && p.carry_out && q.turn == p.tiles - 1) *reinterpret_cast<float2*>(p.carry_out + at) = through(all, in);
  const float2 first = through(pre, in);
  float h0 = first.x, h1 = first.y;
  if (!q.active || q.row0 >= p.s) return;
  if (p.saved && q.row0 % kRecSave == 0) {
    const int64_t n_saved = (p.s + kRecSave - 1) / kRecSave;
    *reinterpret_cast<float2*>(p.saved + (q.n * n_saved + q.row0 / kRecSave) * p.h + q.c0) = make_float2(h0, h1);
  }
  const RecRows<T> dst(p.out, p.h, q, p.s, L);
  const int rows = again(lim);
#pragma unroll
  for (int i = 0; i < L; ++i) {
    h0 = fmaf(f[i][0], h0, x[i][0]);
    h1 = fmaf(f[i][1], h1, x[i][1]);
    dst.store(P::pack(h0 * r[i][0], h1 * r[i][1]), i, 0, i < rows);
  }
  if (lim < L) dst.zeros(lim, min(p.s - q.row0, L), 0);
}

template <typename T, int L>
__global__ __launch_bounds__(kRecMaxThreads, 4) void recurrence_bwd_kernel(RecParams p) {
  using P = Pair<T>;
  using Raw = typename P::type;
  // forward maps (A, H of either channel), constants of the backward ones (same factors), window of the look back; then the column sums
  constexpr int W = kRecLanes<T>, S = kRecMaxThreads / W;
  __shared__ float4 maps[S][W], win[S][W], near[kRecBlock][W];
  __shared__ float2 back[S][W];
  __shared__ uint32_t ticket;
  const RecPlace q = place_of<W>(p, &ticket, true, L);
  const int64_t h = p.h, ld = 3 * h, n_saved = (p.s + kRecSave - 1) / kRecSave, at = (int64_t)q.n * h + q.c0;
  const uint32_t gate = (uint32_t)p.h * (uint32_t)sizeof(T);
  const int lim = q.active ? min(q.len - q.row0, L) : 0;
  Raw C[L];
  float f[L][2], u[L][2], up[L][2], ds[L][2];   // f, 1 - f, dO R sigmoid(R), dO times the slope of R sigmoid(R)
  float4 own = make_float4(1.f, 0.f, 1.f, 0.f);
  float2 rev = make_float2(0.f, 0.f), state = make_float2(0.f, 0.f);
  {
    const RecRows<T> src(p.gates, ld, q, p.s, L), top(p.d_o, h, q, p.s, L);
    Raw F[L], R[L], D[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool real = i < lim;
      F[i] = src.load(i, 0, real);
      C[i] = src.load(i, gate, real);
      R[i] = src.load(i, 2 * gate, real);
      D[i] = top.load(i, 0, real);
    }
    // the kept state in front of the 64 rows that this sub's are among
    if (q.active && q.row0 < p.s) state = *reinterpret_cast<const float2*>(p.saved + (q.n * n_saved + q.row0 / kRecSave) * h + q.c0);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const float2 F2 = P::floats(i < lim ? F[i] : P::infinities()), C2 = P::floats(C[i]), R2 = P::floats(R[i]), D2 = P::floats(D[i]);   // past the end: f = 1, the rest 0
      sigmoids<T>(F2.x, f[i][0], u[i][0]);
      sigmoids<T>(F2.y, f[i][1], u[i][1]);
      float s0, s1;
      up[i][0] = D2.x * gate_of<T>(R2.x, s0);
      up[i][1] = D2.y * gate_of<T>(R2.y, s1);
      ds[i][0] = D2.x * s0;
      ds[i][1] = D2.y * s1;
      here(f[i]);
      here(u[i]);
      here(up[i]);
      here(ds[i]);
      own.y = fmaf(f[i][0], own.y, u[i][0] * C2.x);
      own.w = fmaf(f[i][1], own.w, u[i][1] * C2.y);
      own.x *= f[i][0];
      own.z *= f[i][1];
    }
#pragma unroll
    for (int i = L - 1; i >= 0; --i) {
      rev.x = f[i][0] * (up[i][0] + rev.x);
      rev.y = f[i][1] * (up[i][1] + rev.y);
    }
  }
  maps[q.sub][q.lane] = own;
  back[q.sub][q.lane] = rev;
  take_carry<W>(p, q, win);
  __syncthreads();
  float4 post = make_float4(1.f, 0.f, 1.f, 0.f);   // of the subs behind
#pragma unroll 2
  for (int j = q.nsub - 1; j > q.sub; --j) {
    const float4 v = maps[j][q.lane];
    const float2 w = back[j][q.lane];
    post = then(post, make_float4(v.x, w.x, v.z, w.y));
  }
  const bool first_sub = q.sub == 0 && q.active;
  const int64_t word = (int64_t)q.turn * p.b * h + at;
  const float4 all = then(post, make_float4(own.x, rev.x, own.z, rev.y));
  if (p.tiles > 1 && first_sub) {
    put_map(p.maps + word, all.x, all.y);
    put_map(p.maps + word + 1, all.z, all.w);
  }
  // forward, while the maps travel: the states, and with them all that does not wait for what comes back: dR, and the factor of g in dF
#pragma unroll 2
  for (int j = q.sub - (q.row0 % kRecSave) / L; j < q.sub; ++j) {   // to the state in front of this sub's rows
    state = through(maps[j][q.lane], state);
  }
  float sum[3][2] = {};
  const RecRows<T> dst(p.out, ld, q, p.s, L);
  int rows = again(lim);
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const float2 C2 = P::floats(C[i]);
    const float s[2] = {state.x, state.y}, c[2] = {C2.x, C2.y};
    float dr[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float now = fmaf(f[i][k], s[k], u[i][k] * c[k]);
      dr[k] = ds[i][k] * now;
      ds[i][k] = (s[k] - c[k]) * (f[i][k] * u[i][k]);
      sum[2][k] += i < rows ? dr[k] : 0.f;   // (behind the last token zero times the state, which may be infinite)
      (k ? state.y : state.x) = now;
    }
    here(ds[i]);
    dst.store(P::pack(dr[0], dr[1]), i, 2 * gate, i < rows);
  }
  const float2 in = look_back<W>(p, q, all, 0, near, win);
  if (first_sub && p.carry_out && q.turn == p.tiles - 1) *reinterpret_cast<float2*>(p.carry_out + at) = through(all, in);
  const float2 behind = through(post, in);
  float B[2] = {behind.x, behind.y};
  rows = again(lim);
#pragma unroll
  for (int i = L - 1; i >= 0; --i) {
    float df[2], dc[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float g = up[i][k] + B[k];
      df[k] = g * ds[i][k];
      dc[k] = g * u[i][k];
      sum[0][k] += i < rows ? df[k] : 0.f;
      sum[1][k] += i < rows ? dc[k] : 0.f;
      B[k] = f[i][k] * g;
    }
    dst.store(P::pack(df[0], df[1]), i, 0, i < rows);
    dst.store(P::pack(dc[0], dc[1]), i, gate, i < rows);
  }
  if (q.active && lim < L)
    for (int m = 0; m < 3; ++m) dst.zeros(lim, min(p.s - q.row0, L), (uint32_t)m * gate);
  if (p.sums) {   // before rounding; the subs' sums leave through LDS
    float2 *red = reinterpret_cast<float2*>(maps), *red2 = reinterpret_cast<float2*>(win);   // two and one of the three
    __syncthreads();
    red[q.sub * W + q.lane] = make_float2(sum[0][0], sum[0][1]);
    red[(S + q.sub) * W + q.lane] = make_float2(sum[1][0], sum[1][1]);
    red2[q.sub * W + q.lane] = make_float2(sum[2][0], sum[2][1]);
    __syncthreads();
    for (int m = q.sub; m < 3; m += q.nsub) {
      const float2* from = m < 2 ? red + m * S * W : red2;
      float2 t = make_float2(0.f, 0.f);
#pragma unroll 2
      for (int j = 0; j < q.nsub; ++j) {
        const float2 v = from[j * W + q.lane];
        t.x += v.x;
        t.y += v.y;
      }
      if (q.active) *reinterpret_cast<float2*>(p.sums + ((int64_t)q.turn * p.b + q.n) * ld + (int64_t)m * h + q.c0) = t;
    }
  }
}

template <typename T> constexpr int kRecRows = 8;   // rows of a sub

struct RecShape { int waves, tiles, rows, groups; int64_t threads; };   // threads: of the launch
template <typename T>
RecShape rec_shape(int b, int s, int h) {
  constexpr int per_wave = kRecRows<T> * 64 / kRecLanes<T>;   // rows
  RecShape r;
  r.groups = ceil_div(h, 2 * kRecLanes<T>);
  r.waves = kRecWaves;
  while (r.waves > 1 && (int64_t)per_wave * r.waves >= 2 * (int64_t)s) r.waves /= 2;
  r.rows = per_wave * r.waves;
  r.tiles = ceil_div(s, r.rows);
  r.threads = (int64_t)r.tiles * b * r.groups * (64 * r.waves);
  return r;
}
constexpr int kRecMinTileRows = 64, kRecMinCols = 64;   // of a tile, where a sequence has more than one

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool rec_ok(const RecurrenceDesc& d) {
  if (d.b <= 0 || d.s <= 0 || d.h <= 0 || d.h % 8 != 0 || (d.dtype != kF32 && d.dtype != kBF16) || (int64_t)d.b * d.s > 0x7fffffff || d.h > (1 << 20))
    return false;
  const RecShape shape = d.dtype == kF32 ? rec_shape<float>(d.b, d.s, d.h) : rec_shape<bf16_t>(d.b, d.s, d.h);
  return shape.threads <= kMaxThreads && recurrence_workspace(d.b, d.s, d.h) > 0 && !(reinterpret_cast<uintptr_t>(d.seqlens) & 3);
}
int64_t rec_max_tiles(int s) { return ((int64_t)s + kRecMinTileRows - 1) / kRecMinTileRows; }

// Workspace, in floats: the tickets, then the words of tiles (8 bytes a channel) and blocks (12), then the column sums.
int64_t rec_tickets(int64_t b, int64_t h) { return b * ((h + kRecMinCols - 1) / kRecMinCols) * kRecTicket; }
int64_t rec_blocks(int64_t tiles) { return (tiles + kRecBlock - 1) / kRecBlock; }
int64_t rec_words(int64_t b, int64_t tiles, int64_t h) { return b * (2 * tiles + 3 * rec_blocks(tiles)) * h; }   // (h: a multiple of 8)

template <typename T, bool BWD>
hipError_t launch_rec(const RecurrenceDesc& d, RecParams p, float* ws, bool sums, hipStream_t s) {
  constexpr int L = kRecRows<T>;
  const RecShape shape = rec_shape<T>(d.b, d.s, d.h);
  p.lens = d.seqlens; p.b = d.b; p.s = d.s; p.h = d.h;
  p.tiles = shape.tiles; p.rows = shape.rows; p.groups = shape.groups;
  // Where rows do not end with a 128-byte line, neighbouring groups share lines, and eight of them in a row go to one XCD's L2; the same where
  // there are 16 chains at most.  us there and back, each on an XCD of its own | so: fp32 32768 x 1000 394 | 369, 2048 x 8200 191 | 176, bf16
  // 32768 x 1000 268 | 240, 32768 x 1024 (8 chains) 236 | 212, 16384 x 2048 (16) 216 | 203.  Other shapes are even within 1 % or lose up to
  // 3 % (fp32 4096 x 4096 160 | 164).
  p.near = (int64_t)d.h * sizeof(T) % 128 != 0 || (int64_t)p.b * p.groups <= 16 ? 8 : 1;
  const int64_t grid = (int64_t)p.tiles * p.b * p.groups;
  const int64_t bh = (int64_t)d.b * d.h;
  const int64_t tickets = rec_tickets(d.b, d.h);
  p.tickets = reinterpret_cast<uint32_t*>(ws);
  p.maps = reinterpret_cast<uint64_t*>(ws + tickets);
  p.block_maps = p.maps + bh * p.tiles;
  p.block_ends = reinterpret_cast<uint32_t*>(p.block_maps + bh * rec_blocks(p.tiles));
  if (sums) p.sums = ws + tickets + rec_words(d.b, p.tiles, d.h);
  if (p.tiles > 1) {
    const int64_t n = rec_words(d.b, p.tiles, d.h) / 4;
    hipLaunchKernelGGL(recurrence_clear_kernel, dim3((unsigned)((tickets / 4 + n + 255) / 256)), dim3(256), 0, s, reinterpret_cast<uint4*>(ws),
                       tickets / 4, n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (BWD) hipLaunchKernelGGL((recurrence_bwd_kernel<T, L>), dim3((unsigned)grid), dim3(64 * shape.waves), 0, s, p);
  else hipLaunchKernelGGL((recurrence_fwd_kernel<T, L>), dim3((unsigned)grid), dim3(64 * shape.waves), 0, s, p);
  return hipGetLastError();
}

}  // namespace

int64_t recurrence_saved(int b, int s, int h) { return (int64_t)b * (((int64_t)s + kRecSave - 1) / kRecSave) * h; }

int64_t recurrence_workspace(int b, int s, int h) {   // column sums [b * tiles][3h] and words of the same size
  const int64_t tiles = rec_max_tiles(s), rows = (int64_t)b * tiles;
  if (rows > (1ll << 33) / h) return 0;   // (over 2^37 bytes)
  return rec_tickets(b, h) + rec_words(b, tiles, h) + 3 * rows * h;
}

hipError_t recurrence_fwd(const RecurrenceDesc& d, const void* gates, const float* state_in, float* state_out, void* o, float* saved,
                          float* workspace, hipStream_t stream) {
  if (!rec_ok(d) || !gates || !o || !workspace || !aligned16(gates) || !aligned16(o) || !aligned16(workspace) || !aligned16(saved) ||
      !aligned16(state_in) || !aligned16(state_out))
    return hipErrorInvalidValue;
  RecParams p{};
  p.gates = gates; p.out = o; p.carry_in = state_in; p.carry_out = state_out; p.saved = saved;
  return d.dtype == kBF16 ? launch_rec<bf16_t, false>(d, p, workspace, false, stream) : launch_rec<float, false>(d, p, workspace, false, stream);
}

hipError_t recurrence_bwd(const RecurrenceDesc& d, const void* gates, const float* saved, const void* d_o, const float* dstate_out,
                          float* dstate_in, void* dgates, float* dbias, bool accumulate, float* workspace, hipStream_t stream) {
  if (!rec_ok(d) || !gates || !saved || !d_o || !dgates || !workspace || !aligned16(gates) || !aligned16(saved) || !aligned16(d_o) ||
      !aligned16(dgates) || !aligned16(workspace) || !aligned16(dstate_out) || !aligned16(dstate_in) || !aligned16(dbias))
    return hipErrorInvalidValue;
  RecParams p{};
  p.gates = gates; p.d_o = d_o; p.out = dgates; p.carry_in = dstate_out; p.carry_out = dstate_in; p.saved = const_cast<float*>(saved);
  const hipError_t e = d.dtype == kBF16 ? launch_rec<bf16_t, true>(d, p, workspace, dbias != nullptr, stream)
                                        : launch_rec<float, true>(d, p, workspace, dbias != nullptr, stream);
  if (e != hipSuccess || !dbias) return e;
  const RecShape shape = d.dtype == kBF16 ? rec_shape<bf16_t>(d.b, d.s, d.h) : rec_shape<float>(d.b, d.s, d.h);
  const FinalizeItem fin{workspace + rec_tickets(d.b, d.h) + rec_words(d.b, shape.tiles, d.h), d.b * shape.tiles, 3 * d.h, 3 * d.h, dbias};
  return colsum_finalize_grouped(&fin, 1, accumulate, stream);
}

}  // namespace k2bw
