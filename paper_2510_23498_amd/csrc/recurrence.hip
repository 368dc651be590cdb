// Gated linear recurrence along a sequence and its backward pass (rampde_recurrence_fwd / _bwd):
//     h_t = h_{t-1} + r_t (x_t - h_{t-1}),  r_t = 1 / (1 + exp(-z_t)).
// The update is written as an increment, as the time stepper's are: an error in r_t then is an error of the rate alone and
// does not move the fixed point h = x, where a h + (1 - a) x would drift by the rounding of a over 1 / (1 - a) steps.
//
// Channels of all samples are one index c = b D + d; a lane owns two of a block of 128, neighbours where a word holds both and where
// channels share a gate (a power of two of them, at most 128: neighbouring lanes of a wavefront).
//
// Memory bounds it (a step and channel: 6 bytes forward and 10 backward in 16 bits, some 8 and 16 flops).  The update is affine in h,
// so steps are split between workgroups: 128 channels and 128 steps each, one pass over the data, and what goes from tile to tile is
// 8 bytes per channel.  States are saved every 16 steps (fp32, an eighth of h in 16 bits) for the backward pass, which recomputes the
// others.  Measured in bf16, kernels alone: 8 x 4096 x 2048 forward 88 us (402 MB + 17 of states: 4.8 TB/s), backward 133 us
// (671 + 17 MB: 5.2 TB/s); 1 x 65536 x 1024 100 and 144 us; a plain copy of that size reaches 5.0 TB/s.  The words between the tiles
// are emptied before (5 us there, 2 us for 7 x 1003 x 1024).  Few tiles are bound by latency: 7 x 1003 x 1024 in f16, gates shared
// by 64, 12 and 19.5 us for 31 and 45 MB; one step of 32 x 2048 4.4 us.  Odd channels, whose accesses are 2 bytes wide: 8 x 4096 x 2047
// 136 and 273 us.
#include <algorithm>
#include <type_traits>
#include "entry.hpp"
#include "element.hpp"

namespace rampde {
namespace {

constexpr int kSeg = 16;               // steps of a wavefront, and between saved states
constexpr int kBlock = 128;            // channels of a wavefront
constexpr int kWaves = 8;              // of a workgroup
constexpr int kTile = kWaves * kSeg;   // steps of a workgroup
constexpr int kWindow = 16;            // tiles of a chain whose effects are handed on one by one (see words_of)
constexpr int kTicket = 16;            // (tickets are in cache lines of their own)

struct RecArgs {
  const void* x;
  const void* z;
  const float* h0;
  const int32_t* lengths;
  void* h;           // backward: dh
  float* hT;         // backward: dhT
  float* states;     // [segments][B D]
  void* dx;
  void* dz;
  float* dh0;
  int64_t T;
  uint32_t NC, D, share, blocks;
  int tiles;
  int64_t xs[2], zs[2], hs[2];
  uint32_t* tickets;     // tiles > 1: one per block of channels, kTicket apart
  uint64_t* words;       // tiles > 1: [tiles][NC]
};

typedef float f32x2 __attribute__((ext_vector_type(2)));

// The two channels of a lane, GAP apart.  Lanes past the last channel repeat the last ones and store nothing.  PAIR: both are of one
// sample.
template <bool PAIR, int GAP>
struct Lane {
  uint32_t c0;
  bool live0, live1_;
  int n0, n1_;  // steps of their samples
  __device__ inline uint32_t c(int i) const { return i == 0 || live1_ || PAIR ? c0 + i * GAP : c0; }
  __device__ inline bool live(int i) const { return PAIR || i == 0 ? live0 : live1_; }
  __device__ inline int n(int i) const { return PAIR || i == 0 ? n0 : n1_; }
};
__device__ inline int steps_of(const RecArgs& g, uint32_t c) {
  const int T = (int)g.T;
  if (!g.lengths) return T;
  const int len = g.lengths[c / g.D];
  return len < 0 ? 0 : len < T ? len : T;
}
template <int GAP>
__device__ inline uint32_t first_channel() {
  return (GAP == 1 ? 2 : 1) * (threadIdx.x & 63);
}
template <bool PAIR, int GAP>
__device__ inline Lane<PAIR, GAP> lane_of(const RecArgs& g, uint32_t block) {
  Lane<PAIR, GAP> l;
  const uint32_t c = block * kBlock + first_channel<GAP>();
  l.live0 = c < g.NC;
  l.live1_ = c + GAP < g.NC;
  const uint32_t last = PAIR ? g.NC - 2 : g.NC - 1;
  l.c0 = c < last ? c : last;
  l.n0 = l.live0 ? steps_of(g, l.c0) : 0;
  l.n1_ = PAIR ? l.n0 : l.live1_ ? steps_of(g, l.c0 + GAP) : 0;
  return l;
}

// The address as a value of the scalar unit that the compiler does not look into.  (Otherwise it adds the lane's offset to the
// tensor's base once and the row's to that, and every load of a step has a 64-bit address of its own in vector registers.)
__device__ inline uint64_t scalar_address(const void* p) {
  uint64_t a = (uint64_t)(uintptr_t)p;
#ifdef __HIP_DEVICE_COMPILE__
  asm("" : "+s"(a));
#endif
  return a;
}

// How a lane's two channels are reached.  kPairs: one aligned word, through a buffer descriptor at the wavefront's first row: a scalar
// offset of the row and a 32-bit one of the lane, so that an access takes neither vector registers nor vector instructions for its
// address.  kSingles: two elements, likewise (an odd number of channels, odd pitches).  kFar: two elements at 64-bit offsets.
enum Reach { kPairs, kSingles, kFar };
// Elements by themselves are a lane's channels 64 apart, so that an access of the wavefront is a run of 64 neighbours, unless pairs
// share a gate.
template <int REACH, bool SHARED>
constexpr int lane_gap() {
  return REACH == kPairs || SHARED ? 1 : 64;
}

// A wavefront's rows of one tensor, from step t0 (or the last one, where t0 is past the end) on.
struct Window {
  __amdgpu_buffer_rsrc_t r;
};
__device__ inline Window window_of(void* p) { return {__builtin_amdgcn_make_buffer_rsrc(p, 0, -1, 0x00020000)}; }
__device__ inline uint16_t load_b16(const Window& w, uint32_t lane, uint32_t row) {
  return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(w.r, (int)lane, (int)row, 0);
}
__device__ inline uint32_t load_b32(const Window& w, uint32_t lane, uint32_t row) {
  return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(w.r, (int)lane, (int)row, 0);
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ inline u32x2 load_b64(const Window& w, uint32_t lane, uint32_t row) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(w.r, (int)lane, (int)row, 0));
}
__device__ inline void store_b16(const Window& w, uint32_t lane, uint32_t row, uint16_t v) {
  __builtin_amdgcn_raw_buffer_store_b16(v, w.r, (int)lane, (int)row, 0);
}
__device__ inline void store_b32(const Window& w, uint32_t lane, uint32_t row, uint32_t v) {
  __builtin_amdgcn_raw_buffer_store_b32(v, w.r, (int)lane, (int)row, 0);
}
__device__ inline void store_b64(const Window& w, uint32_t lane, uint32_t row, u32x2 v) {
  __builtin_amdgcn_raw_buffer_store_b64(v, w.r, (int)lane, (int)row, 0);
}

template <class T, int REACH, int GAP>
struct Rows {
  typedef typename Elem<T>::S S;
  typedef S S2 __attribute__((ext_vector_type(2)));
  static constexpr bool WIDE = sizeof(S) == 4, PAIR = REACH == kPairs;
  Window win;       // not kFar
  uint32_t off[2];  // bytes
  S* base;          // kFar: row t0 (or the last one)
  int64_t at[2];
  int64_t step;     // elements (not kFar: bytes)
  int left;         // rows behind t0
  __device__ inline Rows(const void* p, const int64_t (&s)[2], const RecArgs& g, const Lane<PAIR, GAP>& l, uint32_t block, uint32_t per, int t0) {
    base = (S*)const_cast<void*>(p);
    const int first_row = t0 < (int)g.T ? t0 : (int)g.T - 1;
    left = (int)g.T - 1 - first_row;
#pragma unroll
    for (int i = 0; i < (PAIR ? 1 : 2); ++i) {
      const uint32_t c = l.c(i), b = c / g.D, d = c - b * g.D;
      at[i] = (int64_t)b * s[0] + d / per;
    }
    if (REACH != kFar) {
      const uint32_t f = block * kBlock, fb = __builtin_amdgcn_readfirstlane(f / g.D), fd = f - fb * g.D;
      const int64_t first = (int64_t)fb * s[0] + __builtin_amdgcn_readfirstlane(fd / per);
      win = window_of(base + first + first_row * s[1]);
      step = s[1] * (int64_t)sizeof(S);
#pragma unroll
      for (int i = 0; i < (PAIR ? 1 : 2); ++i) off[i] = (uint32_t)((at[i] - first) * (int64_t)sizeof(S));
    } else {
      base += first_row * s[1];
      step = s[1];
    }
  }
  __device__ inline S get(int k, int i) const {
    if constexpr (REACH == kFar) return base[k * step + at[i]];
    else if constexpr (WIDE) return __builtin_bit_cast(S, load_b32(win, off[i], (uint32_t)k * (uint32_t)step));
    else return load_b16(win, off[i], (uint32_t)k * (uint32_t)step);
  }
  __device__ inline void put(int k, int i, float v) const {
    if constexpr (REACH == kFar) base[k * step + at[i]] = Elem<T>::down(v);
    else if constexpr (WIDE) store_b32(win, off[i], (uint32_t)k * (uint32_t)step, __builtin_bit_cast(uint32_t, v));
    else store_b16(win, off[i], (uint32_t)k * (uint32_t)step, Elem<T>::down(v));
  }
  // rows past the end: the last one
  __device__ inline S2 load2(int k) const {
    k = k < left ? k : left;
    if constexpr (PAIR && WIDE) return __builtin_bit_cast(S2, load_b64(win, off[0], (uint32_t)k * (uint32_t)step));
    else if constexpr (PAIR) return __builtin_bit_cast(S2, load_b32(win, off[0], (uint32_t)k * (uint32_t)step));
    else return S2{get(k, 0), get(k, 1)};
  }
  __device__ inline S load1(int k) const { return get(k < left ? k : left, 0); }
  __device__ inline void store2(int k, float a, float b, const Lane<PAIR, GAP>& l) const {
    if constexpr (PAIR) {
      if (!l.live(0)) return;
      if constexpr (WIDE) store_b64(win, off[0], (uint32_t)k * (uint32_t)step, __builtin_bit_cast(u32x2, f32x2{a, b}));
      else store_b32(win, off[0], (uint32_t)k * (uint32_t)step, Low<T>::pack2(a, b));
    } else {
      if (l.live(0)) put(k, 0, a);
      if (l.live(1)) put(k, 1, b);
    }
  }
  __device__ inline void store1(int k, float a) const { put(k, 0, a); }
  template <bool SHARED>
  __device__ inline void load_steps(S2 (&v)[kSeg]) const {
#pragma unroll
    for (int k = 0; k < kSeg; ++k) {
      if (SHARED) v[k][0] = load1(k);
      else v[k] = load2(k);
    }
  }
};

// ---- What tiles tell one another.  A chain's tiles are numbered as it runs, and go in windows of kWindow.  A tile has one word per
// channel, all ones until it has something to say.  A chain's first tile and every window's last say {0, H}: the state behind them.
// The others say {A, U}: they take a state h to A h + U (A is a product of factors 1 - r in [0, 1], or a NaN).  The state in front of a
// tile is that behind the window before (the first tile), taken through the window's tiles one after the other: what is added to what
// does not depend on who was first, and two calls give the same bits.  A word is written once and read as a whole (64-bit atomics of
// device scope), so nothing depends on the order of other stores.  The first tile alone reads the state that the caller gives, and its
// word is made of what it read: the last tile, whose state is made of that word, may write over it (hT = h0, dh0 = dhT).  A chain advances by a window in 1.5 us: one alone over 65536 steps takes 49 us, which
// windows of 32 tiles shorten to 39 while 8 x 4096 x 2048 goes from 95 to 100 us.
//
// Every wait ends: a workgroup draws its tile by a ticket of its chain (block of channels), in the order of the chain, so that the
// workgroups it waits for have drawn theirs before and are running; the first tile waits for none, tiles say {A, U} before they wait,
// and a window's last waits for tiles before it alone.  (One ticket for all chains: the draws of 512 workgroups then follow one another, 17 instead of 13 us for
// 7 x 1003 x 1024.)
__device__ inline uint64_t word_of(float a, float u) {
  if (a != a) a = NAN;  // (not the pattern of an empty word)
  return (uint64_t)__builtin_bit_cast(uint32_t, u) << 32 | __builtin_bit_cast(uint32_t, a);
}
typedef __attribute__((address_space(1))) uint64_t global_word;
// (lanes past the last channel never get to their words)
template <int GAP>
__device__ inline global_word* words_of(const RecArgs& g, uint32_t block, int tile) {
  return (global_word*)scalar_address(g.words + (size_t)tile * g.NC + (size_t)block * kBlock) + first_channel<GAP>();
}
template <bool PAIR, int GAP>
__device__ inline void publish(const RecArgs& g, const Lane<PAIR, GAP>& l, uint32_t block, int tile, f32x2 a, f32x2 u) {
  global_word* const mine = words_of<GAP>(g, block, tile);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (l.live(i)) __hip_atomic_store(mine + i * GAP, word_of(a[i], u[i]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The words that the state in front of a tile is made of are those of tiles first, ..., tile - 1 of the chain
__device__ inline int first_word(int tile) {
  const int window = tile & ~(kWindow - 1);
  return window ? window - 1 : 0;
}
// This wavefront's share of them, every eighth, to LDS: waits until they are there
template <bool PAIR, int GAP>
__device__ inline void gather_words(const RecArgs& g, const Lane<PAIR, GAP>& l, uint32_t block, int tile, int wave, f32x4 (&said)[kWindow][64]) {
  constexpr int EACH = kWindow / kWaves;
  const int first = first_word(tile), n = tile - first;
  uint64_t w[EACH][2];
  bool missing[EACH];
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    missing[q] = wave + q * kWaves < n;
#pragma unroll
    for (int i = 0; i < 2; ++i) w[q][i] = 0;
  }
  for (;;) {
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      if (!missing[q]) continue;
      global_word* const theirs = words_of<GAP>(g, block, first + wave + q * kWaves);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (l.live(i)) w[q][i] = __hip_atomic_load(theirs + i * GAP, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    bool wait = false;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      missing[q] = missing[q] && __any(w[q][0] == ~(uint64_t)0 || w[q][1] == ~(uint64_t)0);
      wait |= missing[q];
    }
    if (!wait) break;
    __builtin_amdgcn_s_sleep(2);
  }
#pragma unroll
  for (int q = 0; q < EACH; ++q)
    if (wave + q * kWaves < n) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[2 * i] = __builtin_bit_cast(float, (uint32_t)w[q][i]);
        v[2 * i + 1] = __builtin_bit_cast(float, (uint32_t)(w[q][i] >> 32));
      }
      said[wave + q * kWaves][threadIdx.x & 63] = v;
    }
}
// h taken through n of {A, U}, A U pairs of both channels
__device__ inline f32x2 taken_through(const f32x4 (&by)[kWindow][64], int n, f32x2 h) {
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const f32x4 v = by[s][threadIdx.x & 63];
    h[0] = fmaf(v[0], h[0], v[1]);
    h[1] = fmaf(v[2], h[1], v[3]);
  }
  return h;
}

__global__ __launch_bounds__(256) void recurrence_clear(uint64_t* words, int64_t n, uint32_t* tickets, int64_t nt) {
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) words[i] = ~(uint64_t)0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < nt; i += step) tickets[i] = 0;
}

// this workgroup's place: block of channels, and tile in the order of the chain.  From one round of the blocks to the next the
// blocks move on by one: successive workgroups go to the eight dies in turn, and a die whose workgroups all had the same columns of
// long rows would use a few channels of its cache only (65536 x 1024: 118 instead of 104 us).
__device__ inline void draw(const RecArgs& g, uint32_t& block, int& tile) {
  __shared__ uint32_t drawn;
  const uint32_t k = __builtin_amdgcn_readfirstlane(blockIdx.x / g.blocks);  // (a quotient of uniform numbers comes from the vector unit)
  const uint32_t turn = __builtin_amdgcn_readfirstlane(k % g.blocks), b = blockIdx.x - k * g.blocks + turn;
  block = b < g.blocks ? b : b - g.blocks;
  tile = 0;
  if (g.tiles > 1) {
    if (threadIdx.x == 0) drawn = atomicAdd(g.tickets + (size_t)block * kTicket, 1u);
    __syncthreads();
    tile = __builtin_amdgcn_readfirstlane((int)drawn);
  }
}

// Keeps the compiler from working on more than two steps at a time, whose intermediate values would take the registers of a
// wavefront that could be running
__device__ inline void in_order(int k) {
  if (k & 1) __builtin_amdgcn_sched_barrier(0);
}

// Makes the compiler forget that it has unpacked these values before: it would keep the fp32 ones (twice the registers) from one
// pass over the steps to the next
__device__ inline void repack(uint32_t& v) {
#ifdef __HIP_DEVICE_COMPILE__
  asm("" : "+v"(v));
#endif
}
template <class S2>
__device__ inline void repack_steps(S2 (&v)[kSeg]) {
  if constexpr (sizeof(S2) == 4) {
#pragma unroll
    for (int k = 0; k < kSeg; ++k) {
      uint32_t u = __builtin_bit_cast(uint32_t, v[k]);
      repack(u);
      v[k] = __builtin_bit_cast(S2, u);
    }
  }
}

// bits of the steps k >= n of a wavefront
__device__ inline uint32_t steps_past(int n) { return n >= kSeg ? 0u : n <= 0 ? ~0u : ~0u << n; }

// A workgroup owns 128 channels and 128 steps, a wavefront 16 of the steps, all in registers: gates and inputs are read once.  Each
// wavefront forms what its steps do to a state ({A, U}), the first one folds the eight and gets the state in front of the tile,
// and every wavefront then runs its steps from its own.  In 16 bits three workgroups share a compute unit, whose loads, waits and
// stores overlap (with registers for two, 8 x 4096 x 2048 takes 100 us instead of 96, the emptying of the words included).
template <class T, int REACH, bool SHARED>
__global__ __launch_bounds__(64 * kWaves, sizeof(typename Elem<T>::S) == 2 && REACH == kPairs ? 6 : 4) void recurrence_fwd_tile(RecArgs g) {
  constexpr bool PAIR = REACH == kPairs;
  constexpr int GAP = lane_gap<REACH, SHARED>();
  typedef typename Rows<T, REACH, GAP>::S2 S2;
  __shared__ f32x4 seg[kWaves][64];  // {A, U} of both channels
  __shared__ f32x4 said[kWindow][64];
  __shared__ f32x2 start[64];
  uint32_t block;
  int tile;
  draw(g, block, tile);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = __builtin_amdgcn_readfirstlane(blockDim.x >> 6);
  const Lane<PAIR, GAP> l = lane_of<PAIR, GAP>(g, block);
  const int t0 = tile * kTile + wave * kSeg;  // (below 2^31: the grid is)
  const Rows<T, REACH, GAP> xr(g.x, g.xs, g, l, block, 1, t0), zr(g.z, g.zs, g, l, block, g.share, t0);
  float r[kSeg][2];
  S2 x[kSeg];
  {
    S2 z[kSeg];
    zr.template load_steps<SHARED>(z);
    xr.template load_steps<false>(x);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kSeg; ++k) {
      r[k][0] = logistic<T>(Elem<T>::up(z[k][0]));
      r[k][1] = SHARED ? r[k][0] : logistic<T>(Elem<T>::up(z[k][1]));
      in_order(k);
    }
  }
  // Bit k of past[i]: step k is past the end of channel i's sample.  It passes the state by as it is, also one that is not finite.
  const bool whole = !g.lengths && t0 + kSeg <= g.T;
  const uint32_t past[2] = {steps_past(l.n(0) - t0), steps_past(l.n(1) - t0)};
  auto effect = [&](auto whole_c) {
    f32x2 A = {1.f, 1.f}, U = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kSeg; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float u = fmaf(r[k][i], Elem<T>::up(x[k][i]) - U[i], U[i]), a = fmaf(-r[k][i], A[i], A[i]);
        const bool skip = !decltype(whole_c)::value && (past[i] >> k & 1);
        U[i] = skip ? U[i] : u;
        A[i] = skip ? A[i] : a;
        if (i == 1) in_order(k);
      }
    seg[wave][lane] = f32x4{A[0], U[0], A[1], U[1]};
  };
  if (waves > 1 || g.tiles > 1) {
    if (whole) effect(std::true_type{});
    else effect(std::false_type{});
    __syncthreads();
  }
  repack_steps(x);
  const f32x2 none = {0.f, 0.f};
  f32x2 cur, A = {1.f, 1.f}, U = {0.f, 0.f};
  const bool ends_window = (tile & (kWindow - 1)) == kWindow - 1, chained = tile + 1 < g.tiles;
  f32x2 h = none;  // the state in front of the tile
  if (wave == 0 && tile == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) h[i] = g.h0 && l.live(i) ? g.h0[l.c(i)] : 0.f;
  }
  if (wave == 0 && chained) {
    for (int s = 0; s < waves; ++s) {
      const f32x4 v = seg[s][lane];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        U[i] = fmaf(v[2 * i], U[i], v[2 * i + 1]);
        A[i] *= v[2 * i];
      }
    }
    if (tile == 0) publish(g, l, block, tile, none, f32x2{fmaf(A[0], h[0], U[0]), fmaf(A[1], h[1], U[1])});
    else if (!ends_window) publish(g, l, block, tile, A, U);
  }
  if (tile > 0) {
    gather_words(g, l, block, tile, wave, said);
    __syncthreads();
  }
  if (wave == 0) {
    if (tile > 0) h = taken_through(said, tile - first_word(tile), none);
    if (chained && ends_window) publish(g, l, block, tile, none, f32x2{fmaf(A[0], h[0], U[0]), fmaf(A[1], h[1], U[1])});
    start[lane] = h;
  }
  if (waves > 1) __syncthreads();
  cur = start[lane];
  for (int s = 0; s < wave; ++s) {
    const f32x4 v = seg[s][lane];
    cur[0] = fmaf(v[0], cur[0], v[1]);
    cur[1] = fmaf(v[2], cur[1], v[3]);
  }
  if (g.states && t0 < g.T) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (l.live(i)) g.states[(size_t)(t0 / kSeg) * g.NC + l.c(i)] = cur[i];
  }
  const Rows<T, REACH, GAP> hr(g.h, g.hs, g, l, block, 1, t0);
  auto output = [&](auto whole_c, auto store_c) {
    constexpr bool WHOLE = decltype(whole_c)::value;
#pragma unroll
    for (int k = 0; k < kSeg; ++k) {
      float out[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float u = fmaf(r[k][i], Elem<T>::up(x[k][i]) - cur[i], cur[i]);
        const bool skip = !WHOLE && (past[i] >> k & 1);
        cur[i] = skip ? cur[i] : u;
        out[i] = skip ? 0.f : u;
      }
      if (decltype(store_c)::value && (WHOLE || t0 + k < g.T)) hr.store2(k, out[0], out[1], l);
    }
  };
  if (!g.h) whole ? output(std::true_type{}, std::false_type{}) : output(std::false_type{}, std::false_type{});
  else whole ? output(std::true_type{}, std::true_type{}) : output(std::false_type{}, std::true_type{});
  if (g.hT && tile + 1 == g.tiles && wave + 1 == waves) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (l.live(i)) g.hT[l.c(i)] = cur[i];
  }
}

// v of another lane of the 16 that the lane is in
template <int CTRL>
__device__ inline float neighbour(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// Sum of a gate's channels, which are `share` neighbouring channels of the wavefront (two per lane).  Up to 16 lanes by the vector unit's
// own lane moves (pairs, pairs of pairs, then mirrored halves, whose lanes hold equal sums by then), through LDS beyond.
__device__ inline float gate_sum(float a, float b, uint32_t share) {
  float s = a + b;
  if (share >= 4) s += neighbour<0xB1>(s);    // quad_perm 1 0 3 2
  if (share >= 8) s += neighbour<0x4E>(s);    // quad_perm 2 3 0 1
  if (share >= 16) s += neighbour<0x141>(s);  // row_half_mirror
  if (share >= 32) s += neighbour<0x140>(s);  // row_mirror
  if (share >= 64) s += __shfl_xor(s, 16);
  if (share >= 128) s += __shfl_xor(s, 32);
  return s;
}

// A rate as one number that holds the smaller of r and 1 - r to fp32: r, or -(1 - r) for open gates (the sign says which, also of a
// zero).  The backward pass multiplies by both: what an open gate leaves of a gradient is G (1 - r), not what G - G r leaves of it.
// (Two numbers would take 32 registers more, and spill: 286 instead of 133 us for 8 x 4096 x 2048.)
__device__ inline float rate_of(const Gate& v) { return v.e < 1.f ? -(v.e * v.s) : v.s; }
__device__ inline bool is_open(float rate) { return __builtin_bit_cast(int, rate) < 0; }
// (1 - r) v and r v.  (Closed: one rounding, of the difference.  A rounded 1 - r would be off the same way at every step.)
__device__ inline float held(float rate, float v) { return fmaf(-rate, v, is_open(rate) ? 0.f : v); }
__device__ inline float passed(float rate, float v) { return fmaf(rate, v, is_open(rate) ? v : 0.f); }

// The same split, the chain of tiles from the last to the first.  A wavefront recomputes its states from the one saved in front of
// its steps, and keeps of a step its rate and the derivative of its state by the gate.
template <class T, int REACH, bool SHARED>
__global__ __launch_bounds__(64 * kWaves, REACH == kPairs ? 4 : 1) void recurrence_bwd_tile(RecArgs g) {
  constexpr bool PAIR = REACH == kPairs;
  constexpr int GAP = lane_gap<REACH, SHARED>();
  typedef typename Rows<T, REACH, GAP>::S2 S2;
  __shared__ f32x4 seg[kWaves][64];
  __shared__ f32x4 said[kWindow][64];
  __shared__ f32x2 start[64];
  uint32_t block;
  int place;  // in the chain, from the last tile on
  draw(g, block, place);
  const int tile = g.tiles - 1 - place;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = __builtin_amdgcn_readfirstlane(blockDim.x >> 6);
  const Lane<PAIR, GAP> l = lane_of<PAIR, GAP>(g, block);
  const int t0 = tile * kTile + wave * kSeg;  // (below 2^31: the grid is)
  const Rows<T, REACH, GAP> xr(g.x, g.xs, g, l, block, 1, t0), zr(g.z, g.zs, g, l, block, g.share, t0);
  const bool whole = !g.lengths && t0 + kSeg <= g.T;
  const uint32_t past[2] = {steps_past(l.n(0) - t0), steps_past(l.n(1) - t0)};
  float r[kSeg][2], q[kSeg][2];
  S2 dh[kSeg];
  {
    S2 x[kSeg], z[kSeg];
    zr.template load_steps<SHARED>(z);
    xr.template load_steps<false>(x);
    if (g.h) {
      const Rows<T, REACH, GAP> hr(g.h, g.hs, g, l, block, 1, t0);
      hr.template load_steps<false>(dh);
    } else {
#pragma unroll
      for (int k = 0; k < kSeg; ++k) dh[k] = S2{0, 0};
    }
    f32x2 cur = {0.f, 0.f};
    if (t0 < g.T) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (l.live(i)) cur[i] = g.states[(size_t)(t0 / kSeg) * g.NC + l.c(i)];
    }
    __builtin_amdgcn_sched_barrier(0);
    // (steps past the end of a sample come last: what they make of the state and of q is not used)
#pragma unroll
    for (int k = 0; k < kSeg; ++k) {
      r[k][0] = rate_of(gate_of<T>(Elem<T>::up(z[k][0])));
      r[k][1] = SHARED ? r[k][0] : rate_of(gate_of<T>(Elem<T>::up(z[k][1])));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float move = passed(r[k][i], Elem<T>::up(x[k][i]) - cur[i]);
        q[k][i] = held(r[k][i], move);  // r (1 - r) (x - h)
        cur[i] += move;
      }
      in_order(k);
    }
  }
  auto effect = [&](auto whole_c) {
    f32x2 A = {1.f, 1.f}, U = {0.f, 0.f};
#pragma unroll
    for (int k = kSeg - 1; k >= 0; --k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float G = U[i] + Elem<T>::up(dh[k][i]), u = held(r[k][i], G), a = held(r[k][i], A[i]);
        const bool skip = !decltype(whole_c)::value && (past[i] >> k & 1);
        U[i] = skip ? U[i] : u;
        A[i] = skip ? A[i] : a;
        if (i == 1) in_order(k);
      }
    seg[wave][lane] = f32x4{A[0], U[0], A[1], U[1]};
  };
  if (waves > 1 || g.tiles > 1) {
    if (whole) effect(std::true_type{});
    else effect(std::false_type{});
    __syncthreads();
  }
  repack_steps(dh);
  const f32x2 none = {0.f, 0.f};
  f32x2 A = {1.f, 1.f}, U = {0.f, 0.f};
  const bool ends_window = (place & (kWindow - 1)) == kWindow - 1, chained = tile > 0;
  f32x2 h = none;  // what comes to the tile from the steps behind it
  if (wave == 0 && place == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) h[i] = g.hT && l.live(i) ? g.hT[l.c(i)] : 0.f;
  }
  if (wave == 0 && chained) {
    for (int s = waves - 1; s >= 0; --s) {
      const f32x4 v = seg[s][lane];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        U[i] = fmaf(v[2 * i], U[i], v[2 * i + 1]);
        A[i] *= v[2 * i];
      }
    }
    if (place == 0) publish(g, l, block, place, none, f32x2{fmaf(A[0], h[0], U[0]), fmaf(A[1], h[1], U[1])});
    else if (!ends_window) publish(g, l, block, place, A, U);
  }
  if (place > 0) {
    gather_words(g, l, block, place, wave, said);
    __syncthreads();
  }
  if (wave == 0) {
    if (place > 0) h = taken_through(said, place - first_word(place), none);
    if (chained && ends_window) publish(g, l, block, place, none, f32x2{fmaf(A[0], h[0], U[0]), fmaf(A[1], h[1], U[1])});
    start[lane] = h;
  }
  if (waves > 1) __syncthreads();
  f32x2 c = start[lane];  // (1 - r_t) G_t: what goes on to the step before
  for (int s = waves - 1; s > wave; --s) {
    const f32x4 v = seg[s][lane];
    c[0] = fmaf(v[0], c[0], v[1]);
    c[1] = fmaf(v[2], c[1], v[3]);
  }
  const Rows<T, REACH, GAP> dxr(g.dx, g.xs, g, l, block, 1, t0), dzr(g.dz, g.zs, g, l, block, g.share, t0);
  auto output = [&](auto whole_c) {
    constexpr bool WHOLE = decltype(whole_c)::value;
#pragma unroll
    for (int k = kSeg - 1; k >= 0; --k) {
      float gx[2], gz[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float G = c[i] + Elem<T>::up(dh[k][i]);
        const bool skip = !WHOLE && (past[i] >> k & 1);
        gx[i] = skip ? 0.f : passed(r[k][i], G);
        gz[i] = skip ? 0.f : G * q[k][i];
        c[i] = skip ? c[i] : held(r[k][i], G);
      }
      if (!WHOLE && t0 + k >= g.T) continue;
      dxr.store2(k, gx[0], gx[1], l);
      if (SHARED) {
        const float sum = gate_sum(gz[0], gz[1], g.share);
        if (l.live(0) && (l.c0 & (g.share - 1)) == 0) dzr.store1(k, sum);
      } else {
        dzr.store2(k, gz[0], gz[1], l);
      }
      in_order(k);
    }
  };
  if (whole) output(std::true_type{});
  else output(std::false_type{});
  if (g.dh0 && tile == 0 && wave == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (l.live(i)) g.dh0[l.c(i)] = c[i];
  }
}

// strides of [B][T][width] rows, contiguous ones filled in; false where rows would overlap
bool fill_strides(const int64_t (&given)[2], int64_t B, int64_t T, int64_t width, int64_t (&s)[2]) {
  s[0] = given[0];
  s[1] = given[1];
  if (s[0] == 0 && s[1] == 0) {
    s[0] = T * width;
    s[1] = width;
  }
  const int64_t most = (int64_t)1 << 40, end = (int64_t)1 << 46;  // (no tensor reaches these; the products below stay in 64 bits)
  if (s[0] < 0 || s[1] < 0 || s[0] > most || s[1] > most) return false;
  if (s[0] && B - 1 > end / s[0]) return false;
  if (s[1] && T - 1 > end / s[1]) return false;
  if (T > 1 && s[1] < width) return false;
  if (B > 1 && s[0] < width) return false;
  return B == 1 || T == 1 || s[0] >= (T - 1) * s[1] + width || s[1] >= (B - 1) * s[0] + width;
}

unsigned threads_of(int64_t T) { return 64 * (unsigned)std::min<int64_t>(kWaves, (T + kSeg - 1) / kSeg); }

int check(const rampde_recurrence* r, RecArgs& g) {
  if (!r || r->B < 1 || r->T < 1 || r->D < 1 || !known_type(r->low)) return RAMPDE_EINVAL;
  if (r->share < 1 || (r->share & (r->share - 1)) || r->D % r->share) return RAMPDE_EINVAL;
  if (r->share > 128) return RAMPDE_EUNSUPPORTED;
  if (r->T >= (int64_t)1 << 30 || r->B >= (int64_t)1 << 31 || r->D >= (int64_t)1 << 31) return RAMPDE_EUNSUPPORTED;
  if (r->B * r->D > (int64_t)1 << 31) return RAMPDE_EUNSUPPORTED;
  if (!launchable((r->B * r->D + kBlock - 1) / kBlock * ((r->T + kTile - 1) / kTile), threads_of(r->T))) return RAMPDE_EUNSUPPORTED;
  g.T = r->T;
  g.D = (uint32_t)r->D;
  g.NC = (uint32_t)(r->B * r->D);
  g.share = (uint32_t)r->share;
  g.blocks = (g.NC + kBlock - 1) / kBlock;
  g.tiles = (int)((g.T + kTile - 1) / kTile);
  if (!fill_strides(r->x_stride, r->B, r->T, r->D, g.xs) || !fill_strides(r->z_stride, r->B, r->T, r->D / r->share, g.zs) ||
      !fill_strides(r->h_stride, r->B, r->T, r->D, g.hs))
    return RAMPDE_EINVAL;
  return RAMPDE_OK;
}

// how the channels of a tensor can be reached (see Reach)
Reach reach(const void* p, const int64_t (&s)[2], const RecArgs& g, size_t e, uint32_t per) {
  const int64_t samples = std::min<int64_t>(g.NC / g.D, kBlock / g.D + 2);
  if (((samples - 1) * s[0] + g.D + kSeg * s[1]) * (int64_t)e >= (int64_t)1 << 31) return kFar;
  if (per > 1 || !p) return kPairs;  // (one element, shared by the pair)
  const bool even = (g.T == 1 || s[1] % 2 == 0) && (g.D == g.NC || s[0] % 2 == 0);
  return g.D % 2 == 0 && aligned_to(p, 2 * e) && even ? kPairs : kSingles;
}

size_t ticket_bytes(const RecArgs& g) { return ((size_t)g.blocks * kTicket * 4 + 255) & ~(size_t)255; }
size_t chain_bytes(const RecArgs& g) {
  return g.tiles > 1 ? ticket_bytes(g) + (((size_t)g.tiles * g.NC * 8 + 255) & ~(size_t)255) : 256;
}

template <bool BACK, class T, int REACH>
void launch_tile(const RecArgs& g, hipStream_t st) {
  const unsigned grid = g.blocks * (unsigned)g.tiles;
  const unsigned threads = threads_of(g.T);
  if constexpr (BACK) {
    if (g.share > 1) recurrence_bwd_tile<T, REACH, true><<<grid, threads, 0, st>>>(g);
    else recurrence_bwd_tile<T, REACH, false><<<grid, threads, 0, st>>>(g);
  } else {
    if (g.share > 1) recurrence_fwd_tile<T, REACH, true><<<grid, threads, 0, st>>>(g);
    else recurrence_fwd_tile<T, REACH, false><<<grid, threads, 0, st>>>(g);
  }
}

template <bool BACK>
int run(RecArgs& g, rampde_dtype low, void* workspace, hipStream_t st) {
  if (g.tiles > 1) {
    g.tickets = (uint32_t*)workspace;
    g.words = (uint64_t*)((char*)workspace + ticket_bytes(g));
    const int64_t n = (int64_t)g.tiles * g.NC;
    recurrence_clear<<<(unsigned)std::min<int64_t>((n + 1023) / 1024, 2048), 256, 0, st>>>(g.words, n, g.tickets,
                                                                                          (int64_t)g.blocks * kTicket);
    HIP_TRY(hipGetLastError());
  }
  const size_t e = type_size(low);
  int far = std::max({reach(g.x, g.xs, g, e, 1), reach(g.z, g.zs, g, e, g.share), reach(g.h, g.hs, g, e, 1)});
  if (BACK) far = std::max<int>({far, reach(g.dx, g.xs, g, e, 1), reach(g.dz, g.zs, g, e, g.share)});
  return by_type(low, [&](auto tag) {
    typedef decltype(tag) T;
    if (far == kPairs) launch_tile<BACK, T, kPairs>(g, st);
    else if (far == kSingles) launch_tile<BACK, T, kSingles>(g, st);
    else launch_tile<BACK, T, kFar>(g, st);
    HIP_TRY(hipGetLastError());
    return (int)RAMPDE_OK;
  });
}

}  // namespace
}  // namespace rampde

using namespace rampde;

extern "C" {

int64_t rampde_recurrence_states(const rampde_recurrence* r) {
  RecArgs g{};
  return check(r, g) == RAMPDE_OK ? (g.T + kSeg - 1) / kSeg * (int64_t)g.NC : 0;
}

size_t rampde_recurrence_workspace_bytes(const rampde_recurrence* r) {
  RecArgs g{};
  return check(r, g) == RAMPDE_OK ? chain_bytes(g) : 0;
}

int rampde_recurrence_fwd(const rampde_recurrence* r, const void* x, const void* z, const float* h0, const int32_t* lengths,
                          void* h, float* hT, float* states, void* workspace, size_t workspace_bytes, void* hip_stream) {
  RecArgs g{};
  if (const int rc = check(r, g)) return rc;
  const size_t e = type_size(r->low);
  if (!x || !z || !aligned_to(x, e) || !aligned_to(z, e) || !aligned_to(h, e) || !aligned_to(h0, 4) || !aligned_to(hT, 4) ||
      !aligned_to(states, 4) || !aligned_to(lengths, 4))
    return RAMPDE_EINVAL;
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < chain_bytes(g)) return RAMPDE_EWORKSPACE;
  g.x = x, g.z = z, g.h0 = h0, g.lengths = lengths, g.h = h, g.hT = hT, g.states = states;
  return run<false>(g, r->low, workspace, (hipStream_t)hip_stream);
}

int rampde_recurrence_bwd(const rampde_recurrence* r, const void* x, const void* z, const int32_t* lengths, const float* states,
                          const void* dh, const float* dhT, void* dx, void* dz, float* dh0, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  RecArgs g{};
  if (const int rc = check(r, g)) return rc;
  const size_t e = type_size(r->low);
  if (!x || !z || !states || !dx || !dz || !aligned_to(x, e) || !aligned_to(z, e) || !aligned_to(dh, e) || !aligned_to(dx, e) ||
      !aligned_to(dz, e) || !aligned_to(states, 4) || !aligned_to(dhT, 4) || !aligned_to(dh0, 4) || !aligned_to(lengths, 4))
    return RAMPDE_EINVAL;
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < chain_bytes(g)) return RAMPDE_EWORKSPACE;
  g.x = x, g.z = z, g.lengths = lengths, g.states = const_cast<float*>(states), g.h = const_cast<void*>(dh);
  g.hT = const_cast<float*>(dhT), g.dx = dx, g.dz = dz, g.dh0 = dh0;
  return run<true>(g, r->low, workspace, (hipStream_t)hip_stream);
}

}  // extern "C"
