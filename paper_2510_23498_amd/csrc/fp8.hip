// Matrix product in 8-bit floating point with a power-of-two scale for every 128 values along the contraction
// (rampde_fp8_quantize, rampde_fp8_matmul, rampde_fp8_matmul_short).
//
// Sums in fp32 (rampde_fp8_matmul, any result): an e4m3 value times its scale is a bf16 number, one instruction converts two of
// them, and 16-bit matrix instructions form exact products and fp32 sums (5e-9 relative on blocks of 128 normally distributed values
// against 64 bits, 8e-8 on values spread over all exponents).  e4m3 goes down to 2^-9, scales to 2^-127 and bf16 to 2^-133 only (gradients
// that die away along a sequence do get there): operands are converted with three more in the exponent, and the sums take it back.
// Values past 2^124 and sums past 2^122, which then have no room above, take short sums.
//
// Short sums (rampde_fp8_matmul_short, results of 16 bits; a caller has to ask for them): gfx950's scaled matrix instructions multiply
// the 8-bit values and apply an exponent per operand row and 32 values, so that a scale that is a power of two costs nothing, at twice
// the rate.  They (scaled or not) align 8 products that follow one another along the contraction to the largest of them and drop what
// is more than 13 binary places below its leading one; from one such group to the next, and to the accumulator, they keep 24 bits.  A
// sum of eight is off by at most 7 * 2^-13 of its largest product: 1.5e-5 and 4.9e-5 on the same blocks, which flips the rounding of
// enough results that they differ from those of fp32 sums by 1e-4 to 3e-4 norm-wise.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "entry.hpp"
#include "element.hpp"

namespace rampde {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// ------------------------------------------------------------------ quantisation
// Exponent of the smallest power of two, at least 2^-127, with which |v| <= top stays within 448 = 0.875 * 2^9.
__device__ inline int scale_exponent(float top) {
  if (!(top > 0.f)) return 0;
  int k;
  const float m = frexpf(top, &k);
  const int e = m <= 0.875f ? k - 9 : k - 8;
  return e < -127 ? -127 : e;
}
__device__ inline float finite_magnitude(float v) {
  const float a = fabsf(v);
  return a < INFINITY ? a : 0.f;  // (a NaN compares false)
}
__device__ inline float to_nan(float v) { return fabsf(v) < INFINITY ? v : NAN; }  // e4m3 has no infinities
// four values (none infinite), each times 2^-e, as bytes (nearest even)
__device__ inline uint32_t pack4(float a, float b, float c, float d, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
  return (uint32_t)w;
}
__device__ inline float inverse_scale(int e) { return __builtin_bit_cast(float, (uint32_t)(127 - e) << 23); }

struct QuantArgs {
  const void* src;
  int64_t ld, R, K;
  uint8_t *values, *scales;      // of [R][K]
  uint8_t *values_t, *scales_t;  // of the transpose
  int64_t Kq, Ks, Rq, Rs;        // pitches of values and scales, of either operand
};

// the scale byte of block kb of nb, and the padding behind the last one
__device__ inline void put_scale(uint8_t* row, int64_t kb, int64_t nb, int64_t pitch, int e) {
  row[kb] = (uint8_t)(e + 127);
  if (kb == nb - 1)
    for (int64_t i = nb; i < pitch; ++i) row[i] = 127;
}

// 16 lanes per block of 128 columns of a row, 8 values each; four neighbouring blocks of a row per lane, so that enough loads are on
// their way.  grid (rows / 16, blocks / 4).  The largest magnitude is that of the bit patterns, which order infinities and NaN above
// every number: only where it is one of them are finite values looked for apart.  Memory bounds it (2 bytes in, 1 out and an eighth of a
// percent of scales): 16384 x 4096 in bf16 41 us, 4.9 TB/s; 16 rows of 2048 3.6 us.
constexpr int kRowBlocks = 4;
template <class T>
__global__ __launch_bounds__(256) void quantize_rows(QuantArgs g) {
  typedef typename Elem<T>::S S;
  const int64_t nb = g.Kq / 128, row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int kb0 = blockIdx.y * kRowBlocks, lane8 = (threadIdx.x & 15) * 8;
  if (row >= g.R) return;
  Raw8<T> raw[kRowBlocks];
  const S* p = (const S*)g.src + row * g.ld;
#pragma unroll
  for (int j = 0; j < kRowBlocks; ++j) {
    const int64_t c = (int64_t)(kb0 + j) * 128 + lane8;
    const int n = g.K - c < 0 ? 0 : g.K - c < 8 ? (int)(g.K - c) : 8;
    raw[j] = load8<T>(p + c, n);
  }
#pragma unroll
  for (int j = 0; j < kRowBlocks; ++j) {
    if (kb0 + j >= nb) return;
    float v[8];
    unpack8<T>(raw[j], v);
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = __builtin_bit_cast(uint32_t, v[i]) & 0x7FFFFFFFu;
      bits = bits > u ? bits : u;
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const uint32_t u = (uint32_t)__shfl_xor((int)bits, o);
      bits = bits > u ? bits : u;
    }
    float top = __builtin_bit_cast(float, bits);
    if (bits >= 0x7F800000u) {  // (the same for all lanes of the block)
      top = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top = fmaxf(top, finite_magnitude(v[i]));
        v[i] = to_nan(v[i]);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    }
    const int e = scale_exponent(top);
    const float inv = inverse_scale(e);
    uint2 w;
    w.x = pack4(v[0], v[1], v[2], v[3], inv);
    w.y = pack4(v[4], v[5], v[6], v[7], inv);
    *reinterpret_cast<uint2*>(g.values + row * g.Kq + (int64_t)(kb0 + j) * 128 + lane8) = w;
    if (lane8 == 0) put_scale(g.scales + row * g.Ks, kb0 + j, nb, g.Ks, e);
  }
}

// A tile of 128 x 128 of the source: thread (tr, tc) has RT rows from RT tr on, 8 columns from 8 tc on.  BLOCKS: one scale for the tile, both
// operands; else a scale per column, the transpose alone.  The tile is turned in LDS, so that both sides see whole rows of 128 bytes
// (or more): columns of 16384 x 4096 in bf16 33 us from a warm last-level cache, 47 from memory (4.3 TB/s), blocks of 4096 x 2048 in
// fp32 with both operands 10 and 13 us.
template <class T, bool BLOCKS, int RT>
__global__ __launch_bounds__(16 * 128 / RT) void quantize_tile(QuantArgs g) {
  typedef typename Elem<T>::S S;
  constexpr int THREADS = 16 * 128 / RT, WAVES = THREADS / 64;
  __shared__ __attribute__((aligned(16))) float tops[WAVES][128];  // of the wavefronts' rows
  // The transposed tile, 128 bytes per column in 16 chunks of 8 rows; chunk i of a column is in place i ^ place(column), which spreads
  // the wavefront's writes (columns 8 apart) and reads (neighbouring columns) over the banks.
  __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
  auto place = [](int col) { return ((col >> 3) ^ (col >> 1)) & 15; };
  const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)blockIdx.y * 128, c0 = (int64_t)blockIdx.x * 128;
  const int64_t c = c0 + tc * 8;
  const int n = g.K - c < 0 ? 0 : g.K - c < 8 ? (int)(g.K - c) : 8;
  Raw8<T> raw[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t row = r0 + tr * RT + i;
    const S* p = (const S*)g.src + row * g.ld + c;
    const int m = row < g.R ? n : 0;
    raw[i] = load8<T>(p, m);
  }
  float v[RT][8];
#pragma unroll
  for (int i = 0; i < RT; ++i) unpack8<T>(raw[i], v[i]);
  // as in quantize_rows: the largest bit pattern, finite values apart only where one is infinite or NaN
  float top[8];
  bool finite = true;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const uint32_t u = __builtin_bit_cast(uint32_t, v[i][j]) & 0x7FFFFFFFu;
      bits = bits > u ? bits : u;
    }
    finite = finite && bits < 0x7F800000u;
    top[j] = __builtin_bit_cast(float, bits);
  }
  if (!__all(finite)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      top[j] = 0.f;
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        top[j] = fmaxf(top[j], finite_magnitude(v[i][j]));
        v[i][j] = to_nan(v[i][j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    top[j] = fmaxf(top[j], __shfl_xor(top[j], 16));
    top[j] = fmaxf(top[j], __shfl_xor(top[j], 32));
  }
  int e[8];
  if (BLOCKS) {
    float m = top[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) m = fmaxf(m, top[j]);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    if ((threadIdx.x & 63) == 0) tops[0][wave] = m;
    __syncthreads();
    m = tops[0][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, tops[0][w]);
    e[0] = scale_exponent(m);
#pragma unroll
    for (int j = 1; j < 8; ++j) e[j] = e[0];
  } else {
    if ((threadIdx.x & 63) < 16) {
      *reinterpret_cast<f32x4*>(&tops[wave][tc * 8]) = f32x4{top[0], top[1], top[2], top[3]};
      *reinterpret_cast<f32x4*>(&tops[wave][tc * 8 + 4]) = f32x4{top[4], top[5], top[6], top[7]};
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 m = *reinterpret_cast<const f32x4*>(&tops[0][tc * 8 + 4 * h]);
#pragma unroll
      for (int w = 1; w < WAVES; ++w) {
        const f32x4 o = *reinterpret_cast<const f32x4*>(&tops[w][tc * 8 + 4 * h]);
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = fmaxf(m[j], o[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) e[4 * h + j] = scale_exponent(m[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float inv = inverse_scale(e[j]);
    const int col = tc * 8 + j;
#pragma unroll
    for (int h = 0; h < RT; h += 4) {
      const int at = tr * RT + h;  // byte of the column
      *reinterpret_cast<uint32_t*>(turned + col * 128 + ((at >> 3) ^ place(col)) * 8 + (at & 7)) =
          pack4(v[h][j], v[h + 1][j], v[h + 2][j], v[h + 3][j], inv);
    }
  }
  const int64_t nb_t = g.Rq / 128, nb = g.Kq / 128;
  if (tr == 0)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) put_scale(g.scales_t + (c + j) * g.Rs, blockIdx.y, nb_t, g.Rs, e[j]);
  if (BLOCKS) {
    const float inv = inverse_scale(e[0]);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t row = r0 + tr * RT + i;
      if (row >= g.R) continue;
      uint2 w;
      w.x = pack4(v[i][0], v[i][1], v[i][2], v[i][3], inv);
      w.y = pack4(v[i][4], v[i][5], v[i][6], v[i][7], inv);
      *reinterpret_cast<uint2*>(g.values + row * g.Kq + c) = w;
      if (tc == 0) put_scale(g.scales + row * g.Ks, blockIdx.x, nb, g.Ks, e[0]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 1024 / THREADS; ++k) {  // 16 bytes each
    const int at = threadIdx.x + THREADS * k, col = at >> 3, part = at & 7;
    if (c0 + col >= g.K) continue;
    const uint2 a = *reinterpret_cast<const uint2*>(turned + col * 128 + ((2 * part) ^ place(col)) * 8);
    const uint2 b = *reinterpret_cast<const uint2*>(turned + col * 128 + ((2 * part + 1) ^ place(col)) * 8);
    *reinterpret_cast<uint4*>(g.values_t + (c0 + col) * g.Rq + r0 + part * 16) = uint4{a.x, a.y, b.x, b.y};
  }
}

// ------------------------------------------------------------------ product
struct Fp8Args {
  const uint8_t *a, *sa, *b, *sb;
  void* c;
  int64_t M, N, ldc;
  int64_t Kq, Ks;
  int nb;          // blocks of 128 along the contraction
  int accumulate;
  bool vec;        // rows of C are 16-byte aligned
  int tiles_m, tiles_n;
  int splits, split_blocks;  // pieces of the contraction (blockIdx.y), blocks of each (a multiple of 4)
  float* part;               // splits > 1: [splits][M][N]
};

// 8 bytes times the scale 2^(e - 127), given as a float, as bf16
__device__ inline u16x8 to_bf16(int lo, int hi, float scale) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  struct { b2 v[4]; } r;
  r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false);
  r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
  r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false);
  r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
  return __builtin_bit_cast(u16x8, r);
}
__device__ inline float scale_value(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
// With kOffset more in the exponent, bf16 holds every e4m3 value (448 at the most) times a scale of up to 2^116 (byte 243).  Whether one of
// these four is larger: a byte of x below n is one that borrows in x - n without having had its upper bit itself.
constexpr uint32_t kOffset = 3;
constexpr float kTakeBack = 1.f / (1 << 2 * kOffset);
__device__ inline bool any_above(uint32_t bytes) { return ((~bytes - 0x0C0C0C0Cu) & bytes & 0x80808080u) != 0; }

template <class T>
__device__ inline void put_c(const Fp8Args& g, int64_t m, int64_t n, f32x4 v) {
  typedef typename Elem<T>::S S;
  if (m >= g.M) return;
  S* p = (S*)g.c + m * g.ldc + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < g.N) {
      float s = v[i];
      if (g.accumulate) s += Elem<T>::up(p[i]);
      p[i] = Elem<T>::down(s);
    }
}

// ---- Few rows of A (up to 32): reading B once is the floor.  A workgroup owns 16 FM rows x 16 columns of C and a piece of the
// contraction, its 16 wavefronts a sixteenth of the piece each, fragments straight from memory, AHEAD blocks requested at a time; the
// sums are added in LDS in the order of the wavefronts.  The first operand of the instruction is B, so that a lane ends with four
// neighbouring columns of a row of C.  A wavefront's load touches 16 rows, a line of each, and that, not the latency, is what bounds
// it: 4 blocks requested at a time took as long.  In cache, 16 x 4096 x 4096 takes 8 us (2.1 TB/s of B), 16 x 4096 x 2048 5 us.
constexpr int kFewWaves = 16;
template <class T, bool SHORT, int FM>
__global__ __launch_bounds__(64 * kFewWaves) void fp8_few_rows(Fp8Args g) {
  constexpr int AHEAD = 2;
  __shared__ f32x4 sums[kFewWaves][FM][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t n = n0 + r < g.N ? n0 + r : g.N - 1;
  const uint8_t* pb = g.b + n * g.Kq + q * 32;
  const uint8_t* qb = g.sb + n * g.Ks;
  const uint8_t *pa[FM], *qa[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t m = 16 * i + r < g.M ? 16 * i + r : g.M - 1;
    pa[i] = g.a + m * g.Kq + q * 32;
    qa[i] = g.sa + m * g.Ks;
  }
  f32x4 acc[FM];
  const int first = (int)blockIdx.y * g.split_blocks, end = first + g.split_blocks < g.nb ? first + g.split_blocks : g.nb;
  const int per = (end - first + kFewWaves - 1) / kFewWaves, k0 = first + wave * per, k1 = k0 + per < end ? k0 + per : end;
  bool above = false;  // (a scale that this lane has met)
  auto sum = [&](auto short_c) {
    constexpr bool NOW_SHORT = decltype(short_c)::value;
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = k0; k < k1; k += AHEAD) {
      i32x8 fa[AHEAD][FM], fb[AHEAD];
      int sa[AHEAD][FM], sb[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int at = k + u < k1 ? k + u : k;
        fb[u] = *reinterpret_cast<const i32x8*>(pb + (int64_t)at * 128);
        sb[u] = qb[at];
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          fa[u][i] = *reinterpret_cast<const i32x8*>(pa[i] + (int64_t)at * 128);
          sa[u][i] = qa[i][at];
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (k + u >= k1) break;
        if constexpr (!NOW_SHORT) {
          static_assert(FM <= 2, "bytes of a word");
          above |= any_above((uint32_t)sb[u] | (uint32_t)sa[u][0] << 8 | (uint32_t)sa[u][FM - 1] << 16);
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const u16x8 wb = to_bf16(fb[u][2 * h], fb[u][2 * h + 1], scale_value(sb[u] + kOffset));
#pragma unroll
            for (int i = 0; i < FM; ++i)
              acc[i] = Low<BF16>::mfma16(wb, to_bf16(fa[u][i][2 * h], fa[u][i][2 * h + 1], scale_value(sa[u][i] + kOffset)), acc[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < FM; ++i)
            acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u], fa[u][i], acc[i], 0, 0, 0, sb[u], 0, sa[u][i]);
        }
      }
    }
  };
  sum(std::integral_constant<bool, SHORT>{});
  if constexpr (!SHORT) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(acc[i][e]));
    if (__any(above || top == INFINITY)) {
      sum(std::true_type{});
    } else {
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[i] *= kTakeBack;
    }
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  if (threadIdx.x < FM * 64) {
    const int i = threadIdx.x >> 6;
    f32x4 s = sums[0][i][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) s += sums[w][i][lane];
    if (g.splits == 1) {
      put_c<T>(g, 16 * i + r, n0 + 4 * q, s);
    } else if (16 * i + r < g.M) {
      float* p = g.part + ((int64_t)blockIdx.y * g.M + 16 * i + r) * g.N + n0 + 4 * q;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n0 + 4 * q + e < g.N) p[e] = s[e];
    }
  }
}

// ---- Tiles.  A workgroup of WM x WN wavefronts owns 32 WM FM rows x 32 WN FN columns of C, a wavefront FM x FN blocks of 32 x 32.
// Blocks of 128 bytes of the rows of both operands (whole cache lines: half lines, a step of 64 at a time, took 10 to 20 % longer) go to
// two LDS slots in turn by direct global->LDS loads; a row's eight 16-byte pieces are permuted (XOR with bits of the row number) so that
// the fragment reads are free of bank conflicts.  One barrier per block, between its halves: the fragments of a block's second half
// are read while the first is multiplied, which frees the slot, and those of the next block's first half while the second is; a block
// has the time of a whole one to arrive.
//
// 256 x 256 on 8 wavefronts (2 x 4, each 128 x 64).  Sums in fp32 are bound by the 16-bit matrix instructions and the conversions in
// front of them: bf16 results 16384 x 4096 x 2048 213 to 255 us and 16384 x 2048 x 4096 205 to 221 us by card and heat (1.1 to 1.35 of
// the 1.8 PFLOP/s that these instructions reach by themselves); 128 x 128 tiles, fp32 results 4096 x 2048 x 16384 219 to 280 us.  Short
// sums: per block of 128, reading fragments from LDS takes as many cycles as the matrix instructions (about 2000 at their full rates), and
// the chip's power lets matrix instructions on such data run at 3.2 to 3.7 PFLOP/s (5 on constant data); the first two products 119 to 151
// and 119 to 154 us (1.8 to 2.3 PFLOP/s).  Tried and slower or no faster, on short sums: 4 wavefronts of 128 x 128, rings of 3 to 5
// half-size slots, tiles of 256 x 128, the 16 x 16 instructions (15 % faster by themselves, but their fragments spill here), wave
// priorities; on fp32 sums: conversions a group ahead.
template <int WM, int WN, int FM, int FN>
struct Fp8Tile {
  static constexpr int TM = 32 * WM * FM, TN = 32 * WN * FN, WAVES = WM * WN;
  static constexpr int SLOT = (TM + TN) * 128;            // bytes
  static constexpr int PERW = (TM + TN) / 8 / WAVES;      // loads of 8 rows per wavefront and block
  static constexpr int PITCH = 64 * FN + 16;              // epilogue: bytes of a staged row of 16-bit results of a wavefront
  static constexpr int STAGE = 32 * FM * PITCH;
  static constexpr int GROUP = 1024 / TM;                 // tile rows that share an XCD's L2 with a few tile columns
  static constexpr int LDS = 2 * SLOT > WAVES * STAGE ? 2 * SLOT : WAVES * STAGE;
};

// 16 bytes of every lane to LDS, lane by lane from `to` on.  (Not a call of the builtin from the template itself: on arguments of
// dependent type the host compilation drops the kernel's launch stub without a word.)
__device__ inline void load_to_lds(const uint8_t* from, __attribute__((address_space(3))) uint8_t* to) {
  __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <class T, bool SHORT, int WM, int WN, int FM, int FN>
__global__ __launch_bounds__(64 * WM * WN, FM * FN > 8 ? 1 : 2) void fp8_tile(Fp8Args g) {
  typedef Fp8Tile<WM, WN, FM, FN> P;
  typedef __attribute__((address_space(3))) uint8_t lds_u8;
  extern __shared__ __attribute__((aligned(16))) uint8_t fp8_smem[];
  lds_u8* ring = (lds_u8*)fp8_smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int frow = lane & 31, half = lane >> 5;
  const int wm = wave / WN, wn = wave % WN;
  // Tiles that run together on an XCD (workgroups go to the eight XCDs in turn) are neighbours: groups of 1024 rows, column by
  // column, so that what they read of both operands is shared in the XCD's L2.
  const int total = g.tiles_m * g.tiles_n;
  int id = blockIdx.x;
  {
    const int per = total / 8, rest = total % 8, xcd = id & 7, at = id >> 3;
    id = xcd * per + (xcd < rest ? xcd : rest) + at;
  }
  const int group = P::GROUP * g.tiles_n, gi = id / group, first = gi * P::GROUP;
  const int rows = g.tiles_m - first < P::GROUP ? g.tiles_m - first : P::GROUP;
  const int64_t m0 = (int64_t)(first + (id - gi * group) % rows) * P::TM, n0 = (int64_t)((id - gi * group) / rows) * P::TN;
  const int kb0 = blockIdx.y * g.split_blocks;
  const int kb1 = kb0 + g.split_blocks < g.nb ? kb0 + g.split_blocks : g.nb;
  const int KT = kb1 - kb0;

  // ---- loader: load i of this wavefront = rows 8 (wave PERW + i) + lane / 8 of the slot (A's, then B's); lane % 8 is the 16-byte
  // place, which holds piece  place ^ ((row >> 1) & 7)
  const int lrow = lane >> 3;
  const uint8_t* base[P::PERW];  // (uniform: a load's 8 rows are of one operand)
  uint32_t off[P::PERW];
#pragma unroll
  for (int i = 0; i < P::PERW; ++i) {
    const int row0 = 8 * (wave * P::PERW + i);
    const bool is_a = row0 < P::TM;
    const int64_t left = (is_a ? g.M - m0 : g.N - n0) - 1;
    const int64_t row = row0 + lrow - (is_a ? 0 : P::TM);
    const int piece = (lane & 7) ^ (((row0 + lrow) >> 1) & 7);
    base[i] = (is_a ? g.a + m0 * g.Kq : g.b + n0 * g.Kq) + (int64_t)kb0 * 128;
    off[i] = (uint32_t)((row < left ? row : left) * g.Kq) + piece * 16;  // (rows past the end: the last one)
  }
  int ld = 0;
  auto issue = [&](int slot_number) {
    lds_u8* slot = ring + slot_number * P::SLOT + wave * P::PERW * 1024;
#pragma unroll
    for (int i = 0; i < P::PERW; ++i) load_to_lds(base[i] + (int64_t)ld * 128 + off[i], slot + i * 1024);
    ld += ld + 1 < KT ? 1 : 0;  // (stays on the last block: the extra loads of the end are in bounds and never multiplied)
  };
  // ---- fragments: of half h of a block a lane has 32 bytes of row frow, pieces 4 h + half and 4 h + 2 + half (the same of both
  // operands, so that the order along the contraction does not matter)
  const int key = (frow >> 1) & 7;
  auto read_frags = [&](int slot_number, int h, i32x8 (&fa)[FM], i32x8 (&fb)[FN]) {
    const lds_u8* slot = ring + slot_number * P::SLOT + frow * 128;
    const int p0 = ((4 * h + half) ^ key) * 16, p1 = ((4 * h + 2 + half) ^ key) * 16;
    auto frag = [&](int row) {
      const i32x4 x = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(slot + row * 128 + p0);
      const i32x4 y = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(slot + row * 128 + p1);
      return i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    };
#pragma unroll
    for (int i = 0; i < (FM > FN ? FM : FN); ++i) {  // (in the order of their use)
      if (i < FN) fb[i] = frag(P::TM + (wn * FN + i) * 32);
      if (i < FM) fa[i] = frag((wm * FM + i) * 32);
    }
  };
  // ---- scales: one register per block of 32 rows holds the bytes of four blocks of 128
  const uint8_t *qa = g.sa + m0 * g.Ks + kb0, *qb = g.sb + n0 * g.Ks + kb0;
  uint32_t oa[FM], ob[FN];
#pragma unroll
  for (int a = 0; a < FM; ++a) {
    const int64_t row = (wm * FM + a) * 32 + frow, left = g.M - m0 - 1;
    oa[a] = (uint32_t)((row < left ? row : left) * g.Ks);
  }
#pragma unroll
  for (int b = 0; b < FN; ++b) {
    const int64_t row = (wn * FN + b) * 32 + frow, left = g.N - n0 - 1;
    ob[b] = (uint32_t)((row < left ? row : left) * g.Ks);
  }
  uint32_t sa[FM], sb[FN], sa_next[FM], sb_next[FN];
  auto load_scales = [&](int k4) {
    const int at = 4 * k4 < kb1 - kb0 ? 4 * k4 : 0;
#pragma unroll
    for (int a = 0; a < FM; ++a) sa_next[a] = *reinterpret_cast<const uint32_t*>(qa + at + oa[a]);
#pragma unroll
    for (int b = 0; b < FN; ++b) sb_next[b] = *reinterpret_cast<const uint32_t*>(qb + at + ob[b]);
  };

  f32x16 acc[FM][FN];
#pragma unroll
  for (int a = 0; a < FM; ++a)
#pragma unroll
    for (int b = 0; b < FN; ++b)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[a][b][q] = 0.f;
  auto multiply = [&](const i32x8 (&fa)[FM], const i32x8 (&fb)[FN]) {
    if constexpr (!SHORT) {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        u16x8 wa[FM], wb[FN];
#pragma unroll
        for (int b = 0; b < FN; ++b) wb[b] = to_bf16(fb[b][2 * h], fb[b][2 * h + 1], scale_value(sb[b] & 255u));
#pragma unroll
        for (int a = 0; a < FM; ++a) wa[a] = to_bf16(fa[a][2 * h], fa[a][2 * h + 1], scale_value(sa[a] & 255u));
#pragma unroll
        for (int a = 0; a < FM; ++a)
#pragma unroll
          for (int b = 0; b < FN; ++b) acc[a][b] = Low<BF16>::mfma32(wb[b], wa[a], acc[a][b]);
      }
    } else {
#pragma unroll
      for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b)
          acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[b], fa[a], acc[a][b], 0, 0, 0, (int)sb[b], 0, (int)sa[a]);
    }
  };

  // reads, requests and arithmetic of half a block go out between its matrix instructions, in whose shadow they then are
  auto spread = [&](auto requests) {
    if constexpr (!SHORT) {
      __builtin_amdgcn_sched_barrier(0);
      return;
    }
    constexpr int NM = FM * FN, READS = 2 * (FM + FN), EACH = (READS + NM - 1) / NM;
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);     // a matrix instruction
      __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);  // fragment reads
      if (decltype(requests)::value) __builtin_amdgcn_sched_group_barrier(0x020, (P::PERW + NM - 1) / NM, 0);
      __builtin_amdgcn_sched_group_barrier(0x006, 5, 0);     // vector and scalar arithmetic
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  i32x8 fa[2][FM], fb[2][FN];
  bool above = false;  // (a scale that this lane has met)
  load_scales(0);
  issue(0);
  issue(1);
#pragma unroll
  for (int a = 0; a < FM; ++a) sa[a] = sa_next[a];
#pragma unroll
  for (int b = 0; b < FN; ++b) sb[b] = sb_next[b];
  static_assert(P::PERW < 64, "vmcnt field");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (P::PERW & 15) | (P::PERW >> 4) << 14);  // vmcnt: block 0 is there
  __builtin_amdgcn_s_barrier();
  read_frags(0, 0, fa[0], fb[0]);
  for (int kb = 0; kb < KT; ++kb) {
    const int slot = kb & 1;
    if ((kb & 3) == 0) {
      if (kb) {
#pragma unroll
        for (int a = 0; a < FM; ++a) sa[a] = sa_next[a];
#pragma unroll
        for (int b = 0; b < FN; ++b) sb[b] = sb_next[b];
      }
      if constexpr (!SHORT) {
#pragma unroll
        for (int a = 0; a < FM; ++a) above |= any_above(sa[a]);
#pragma unroll
        for (int b = 0; b < FN; ++b) above |= any_above(sb[b]);
        // (to four bytes at a time; a byte that carries is one that is above)
#pragma unroll
        for (int a = 0; a < FM; ++a) sa[a] += kOffset * 0x01010101u;
#pragma unroll
        for (int b = 0; b < FN; ++b) sb[b] += kOffset * 0x01010101u;
      }
      load_scales((kb >> 2) + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    read_frags(slot, 1, fa[1], fb[1]);
    multiply(fa[0], fb[0]);
    spread(std::false_type{});
    // This wavefront has read its part of block kb, and its part of block kb + 1 has arrived; after the barrier that is so of all.
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    issue(slot);                           // block kb + 2
    read_frags(slot ^ 1, 0, fa[0], fb[0]); // (past the end: a copy of the last block, never multiplied)
    multiply(fa[1], fb[1]);
    spread(std::true_type{});
#pragma unroll
    for (int a = 0; a < FM; ++a) sa[a] >>= 8;
#pragma unroll
    for (int b = 0; b < FN; ++b) sb[b] >>= 8;
  }
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0), lgkmcnt(0): the end's extra loads and reads
  __builtin_amdgcn_s_barrier();
  // What the offset leaves no room for (see any_above; NaN are none of it): the wavefront sums its blocks of C once more, straight from
  // memory and with the scaled instructions.  That is rare and may be slow; the loop above must not know of it (with both kinds of
  // instructions in it, or with itself a second time behind it, it spills: 2000 and 263 us instead of 211 for 16384 x 4096 x 2048).
  if constexpr (!SHORT) {
    float top = 0.f;
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 16; ++q) top = fmaxf(top, fabsf(acc[a][b][q]));
    above = __any(above || top == INFINITY);
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[a][b][q] *= kTakeBack;
  }
  if (!SHORT && above) {
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[a][b][q] = 0.f;
#pragma unroll 1
    for (int64_t at = (int64_t)kb0 * 128; at < (int64_t)kb1 * 128; at += 64) {  // half a block, of which a lane has 32 bytes
      auto load = [&](const uint8_t* v, const uint8_t* q, int64_t row0, int64_t rows, i32x8& f, int& scale) {
        const int64_t row = row0 + frow < rows ? row0 + frow : rows - 1;
        f = *reinterpret_cast<const i32x8*>(v + row * g.Kq + at + half * 32);
        scale = q[row * g.Ks + (at >> 7)];
      };
      i32x8 w[FN];
      int sw[FN];
#pragma unroll
      for (int b = 0; b < FN; ++b) load(g.b, g.sb, n0 + (wn * FN + b) * 32, g.N, w[b], sw[b]);
#pragma unroll
      for (int a = 0; a < FM; ++a) {
        i32x8 v;
        int sv;
        load(g.a, g.sa, m0 + (wm * FM + a) * 32, g.M, v, sv);
#pragma unroll
        for (int b = 0; b < FN; ++b) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[b], v, acc[a][b], 0, 0, 0, sw[b], 0, sv);
      }
    }
  }

  // ---- accumulator layout of a block: row of C = lane % 32, column = 8 (q / 4) + 4 (lane / 32) + q % 4
  if (g.splits > 1) {
    float* out = g.part + (int64_t)blockIdx.y * g.M * g.N;
#pragma unroll
    for (int a = 0; a < FM; ++a) {
      const int64_t m = m0 + (wm * FM + a) * 32 + frow;
      if (m >= g.M) continue;
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t n = n0 + (wn * FN + b) * 32 + 8 * q + 4 * half;
          float* p = out + m * g.N + n;
          if (n + 4 <= g.N && g.N % 4 == 0) {
            *reinterpret_cast<f32x4*>(p) = f32x4{acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (n + e < g.N) p[e] = acc[a][b][4 * q + e];
          }
        }
    }
    return;
  }
  if constexpr (std::is_same<T, F32>::value) {
#pragma unroll
    for (int a = 0; a < FM; ++a) {
      const int64_t m = m0 + (wm * FM + a) * 32 + frow;
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t n = n0 + (wn * FN + b) * 32 + 8 * q + 4 * half;
          const f32x4 v = {acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
          if (g.vec && m < g.M && n + 4 <= g.N) {
            f32x4* p = reinterpret_cast<f32x4*>((float*)g.c + m * g.ldc + n);
            *p = g.accumulate ? *p + v : v;
          } else {
            put_c<T>(g, m, n, v);
          }
        }
    }
  } else {
    // 16-bit results go through LDS (a region per wavefront) and leave as 16-byte stores of whole row segments
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    lds_u8* stage = ring + wave * P::STAGE;
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(stage + (a * 32 + frow) * P::PITCH + (b * 32 + 8 * q + 4 * half) * 2) =
              u32x2{Low<T>::pack2(acc[a][b][4 * q], acc[a][b][4 * q + 1]), Low<T>::pack2(acc[a][b][4 * q + 2], acc[a][b][4 * q + 3])};
    constexpr int PER_ROW = 4 * FN, ROWS = 64 / PER_ROW;  // lanes of a row, rows of a store
    const int er = lane / PER_ROW, ep = lane % PER_ROW;
    const int64_t n = n0 + wn * FN * 32 + ep * 8;
#pragma unroll 4
    for (int i = 0; i < 32 * FM / ROWS; ++i) {
      const int64_t m = m0 + wm * FM * 32 + i * ROWS + er;
      const u32x4 v = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(stage + (i * ROWS + er) * P::PITCH + ep * 16);
      if (m >= g.M || n >= g.N) continue;
      uint16_t* p = (uint16_t*)g.c + m * g.ldc + n;
      if (g.vec && n + 8 <= g.N) {
        *reinterpret_cast<u32x4*>(p) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e < g.N) p[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// C (+)= the sum of the pieces' shares, in their order
template <class T>
__global__ __launch_bounds__(256) void fp8_fold(Fp8Args g) {
  const int64_t n = g.M * g.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float s = g.part[i];
#pragma unroll 4
    for (int k = 1; k < g.splits; ++k) s += g.part[(int64_t)k * n + i];
    const int64_t m = i / g.N;
    typename Elem<T>::S* p = (typename Elem<T>::S*)g.c + m * g.ldc + (i - m * g.N);
    if (g.accumulate) s += Elem<T>::up(*p);
    *p = Elem<T>::down(s);
  }
}

// ---- which kernel
enum Fp8Kind { kFewRows, kSmallTiles, kLargeTiles };
struct Fp8Plan {
  Fp8Kind kind;
  int splits, split_blocks;
};
Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K) {
  const int nb = (int)((K + 127) / 128);
  auto pieces = [&](Fp8Kind kind, int64_t splits) {  // of a multiple of four blocks each
    const int per = (int)round_up((nb + splits - 1) / splits, 4);
    return Fp8Plan{kind, (nb + per - 1) / per, per};
  };
  const int64_t small = ((M + 127) / 128) * ((N + 127) / 128);
  // (Times of fp32 sums, bf16 results; short sums in brackets where they differ.)
  // Up to 32 rows: tiles of 128 rows take 13 us (10) however few of the rows there are, few-row workgroups 3 to 11 us (M = 16: 3.2 against
  // 6.7 (5.3) us at 512 x 512, 8.4 against 13.9 (11) at 4096 x 4096; M = 32: 11 against 14 (11)).  They fall behind only where the contraction is
  // long and the columns fill the chip as well (M = 16, N = 4096, K = 16384: 24.3 against 23.4 (20)).  Columns that leave compute units
  // idle: the contraction in pieces of at least one block per wavefront (M = 16, N = 1024, K = 8192: 13 us whole, 8 us in four pieces;
  // N = 64, K = 16384: 23 and 7.7 us).
  if (M <= 32) return pieces(kFewRows, std::max<int64_t>(1, std::min<int64_t>(256 / ((N + 15) / 16), nb / 16)));
  // More tiles of 128 x 128 than are resident at two per compute unit: tiles of 256 x 256, which read their operands half as often
  // (4096^3: 101 (59) us, small tiles 120 (74); 16384 x 4096 x 2048: 213 (119) and 231 (148); 2304 x 4096 x 4096: 86 (53) and 84 (60)); with no
  // more, small ones (2048 x 4096 x 4096: 63 (41) us, large tiles 86 (53); 4096 x 2048 x 16384: 216 to 229 and 296).  One large tile occupies a
  // compute unit, and where the last round of them leaves most units idle they lose all the same: 4352 x 4096 x 4096, 272 tiles, 174 (103) us,
  // small tiles 134 to 138 (90); 8448 x 4096 x 2048 140 and 123.
  if (small > 512) return pieces(kLargeTiles, 1);
  // Few small tiles: the contraction in pieces of at least 8 blocks, as long as there is at most one workgroup per compute unit (with up
  // to two: 2048^3 36 (32) us instead of 21 (15), 1024 x 4096 x 4096 49 (39) instead of 38 (30); without pieces 128 x 1024 x 8192 takes 57 (39) us,
  // with 17 (14), 512 x 512 x 4096 31 (22) and 17 (14)).
  return pieces(kSmallTiles, std::max<int64_t>(1, std::min<int64_t>({256 / small, nb / 8, 16})));
}

template <class Kern>
int launch_kernel(Kern kern, const Fp8Args& g, unsigned threads, size_t lds, hipStream_t st) {
  HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  kern<<<dim3((unsigned)(g.tiles_m * g.tiles_n), (unsigned)g.splits), threads, lds, st>>>(g);
  HIP_TRY(hipGetLastError());
  return RAMPDE_OK;
}
template <class T, bool SHORT, int WM, int WN, int FM, int FN>
int launch_tiles(Fp8Args& g, hipStream_t st) {
  typedef Fp8Tile<WM, WN, FM, FN> P;
  g.tiles_m = (int)((g.M + P::TM - 1) / P::TM);
  g.tiles_n = (int)((g.N + P::TN - 1) / P::TN);
  return launch_kernel(fp8_tile<T, SHORT, WM, WN, FM, FN>, g, 64 * P::WAVES, P::LDS, st);
}

bool sizes_ok(int64_t R, int64_t K) { return R >= 1 && K >= 1 && R < (int64_t)1 << 31 && K < (int64_t)1 << 31; }

size_t product_space(int64_t M, int64_t N, const Fp8Plan& p) { return 256 + (p.splits > 1 ? (size_t)p.splits * M * N * 4 : 0); }

int check_product(int64_t M, int64_t N, int64_t K, const void* a_values, const void* a_scales, const void* b_values, const void* b_scales,
                  rampde_dtype c_type, int accumulate, void* C, int64_t ldc, void* workspace, size_t workspace_bytes, Fp8Args& g, Fp8Plan& p) {
  if (!sizes_ok(M, K) || !sizes_ok(N, K) || !known_type(c_type) || !a_values || !a_scales || !b_values || !b_scales || !C) return RAMPDE_EINVAL;
  if (accumulate && c_type != RAMPDE_F32) return RAMPDE_EINVAL;
  if (ldc == 0) ldc = N;
  if (ldc < N || ldc >= (int64_t)1 << 40 || ldc > ((int64_t)1 << 46) / M || !aligned_to(a_values, 16) || !aligned_to(a_scales, 16) || !aligned_to(b_values, 16) ||
      !aligned_to(b_scales, 16) || !aligned_to(C, type_size(c_type)))
    return RAMPDE_EINVAL;
  p = fp8_plan(M, N, K);
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < product_space(M, N, p)) return RAMPDE_EWORKSPACE;
  if (p.kind == kFewRows ? !launchable((N + 15) / 16, 64 * kFewWaves) : !launchable(((M + 255) / 256) * ((N + 255) / 256), 512))
    return RAMPDE_EUNSUPPORTED;  // (small tiles are few)
  if (K >= (int64_t)1 << 23) return RAMPDE_EUNSUPPORTED;  // (offsets of a tile's rows fit 32 bits)
  g.a = (const uint8_t*)a_values, g.sa = (const uint8_t*)a_scales, g.b = (const uint8_t*)b_values, g.sb = (const uint8_t*)b_scales;
  g.c = C, g.M = M, g.N = N, g.ldc = ldc, g.accumulate = accumulate != 0;
  g.Kq = round_up(K, 128), g.nb = (int)(g.Kq / 128), g.Ks = round_up(g.nb, 4);
  g.vec = aligned_to(C, 16) && ldc * (int64_t)type_size(c_type) % 16 == 0;
  g.splits = p.splits, g.split_blocks = p.split_blocks, g.part = (float*)workspace;
  return RAMPDE_OK;
}

template <class T, bool SHORT>
int multiply(Fp8Args& g, const Fp8Plan& p, hipStream_t st) {
  if (p.kind == kFewRows) {
    const dim3 grid((unsigned)((g.N + 15) / 16), (unsigned)g.splits);
    if (g.M <= 16) fp8_few_rows<T, SHORT, 1><<<grid, 64 * kFewWaves, 0, st>>>(g);
    else fp8_few_rows<T, SHORT, 2><<<grid, 64 * kFewWaves, 0, st>>>(g);
    HIP_TRY(hipGetLastError());
  } else if (p.kind == kLargeTiles) {
    if (const int rc = launch_tiles<T, SHORT, 2, 4, 4, 2>(g, st)) return rc;
  } else {
    if (const int rc = launch_tiles<T, SHORT, 2, 2, 2, 2>(g, st)) return rc;
  }
  if (g.splits > 1) {
    fp8_fold<T><<<(unsigned)std::min<int64_t>((g.M * g.N + 255) / 256, 4096), 256, 0, st>>>(g);
    HIP_TRY(hipGetLastError());
  }
  return RAMPDE_OK;
}

}  // namespace
}  // namespace rampde

using namespace rampde;

extern "C" {

int64_t rampde_fp8_value_bytes(int64_t R, int64_t K) { return sizes_ok(R, K) ? R * round_up(K, 128) : 0; }
int64_t rampde_fp8_scale_bytes(int64_t R, int64_t K) { return sizes_ok(R, K) ? R * round_up(round_up(K, 128) / 128, 4) : 0; }

int rampde_fp8_quantize(rampde_dtype src_type, rampde_fp8_mode mode, int64_t R, int64_t K, const void* src, int64_t ld, void* values,
                        void* scales, void* values_t, void* scales_t, void* hip_stream) {
  if (!known_type(src_type) || !sizes_ok(R, K) || !src || !values || !scales) return RAMPDE_EINVAL;
  if (mode != RAMPDE_FP8_ROWS && mode != RAMPDE_FP8_COLS && mode != RAMPDE_FP8_BLOCKS) return RAMPDE_EINVAL;
  if ((mode == RAMPDE_FP8_BLOCKS) != (values_t != nullptr) || (mode == RAMPDE_FP8_BLOCKS) != (scales_t != nullptr)) return RAMPDE_EINVAL;
  if (ld == 0) ld = K;
  const size_t e = type_size(src_type);
  if (ld < K || ld >= (int64_t)1 << 40 || ld > ((int64_t)1 << 46) / R || !aligned_to(src, e) || !aligned_to(values, 16) || !aligned_to(scales, 16) ||
      !aligned_to(values_t, 16) || !aligned_to(scales_t, 16))
    return RAMPDE_EINVAL;
  QuantArgs g{};
  g.src = src, g.ld = ld, g.R = R, g.K = K;
  g.Kq = round_up(K, 128), g.Ks = round_up(g.Kq / 128, 4), g.Rq = round_up(R, 128), g.Rs = round_up(g.Rq / 128, 4);
  g.values = (uint8_t*)values, g.scales = (uint8_t*)scales, g.values_t = (uint8_t*)values_t, g.scales_t = (uint8_t*)scales_t;
  if (mode == RAMPDE_FP8_COLS) g.values_t = g.values, g.scales_t = g.scales;
  const hipStream_t st = (hipStream_t)hip_stream;
  const dim3 row_grid((unsigned)((R + 15) / 16), (unsigned)((g.Kq / 128 + kRowBlocks - 1) / kRowBlocks));
  const dim3 grid((unsigned)(g.Kq / 128), (unsigned)(g.Rq / 128));
  if (mode == RAMPDE_FP8_ROWS ? row_grid.y > 65535 || !launchable(row_grid.x, 256) : grid.y > 65535 || !launchable(grid.x, 512))
    return RAMPDE_EUNSUPPORTED;
  return by_type(src_type, [&](auto tag) {
    typedef decltype(tag) T;
    if (mode == RAMPDE_FP8_ROWS) {
      quantize_rows<T><<<row_grid, 256, 0, st>>>(g);
    } else {
      // Four rows a thread, except for columns of 16 bits in many tiles: 16384 x 4096 in bf16 39 us with four rows, 33 with eight, of 1000 x
      // 1000 5.1 and 6.0; blocks 43 and 47, fp32 columns 64 and 65.
      const bool many = e == 2 && (int64_t)grid.x * grid.y >= 256;
      if (mode == RAMPDE_FP8_BLOCKS) {
        quantize_tile<T, true, 4><<<grid, 512, 0, st>>>(g);
      } else if (many) {
        quantize_tile<T, false, 8><<<grid, 256, 0, st>>>(g);
      } else {
        quantize_tile<T, false, 4><<<grid, 512, 0, st>>>(g);
      }
    }
    HIP_TRY(hipGetLastError());
    return (int)RAMPDE_OK;
  });
}

size_t rampde_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (!sizes_ok(M, K) || !sizes_ok(N, K)) return 0;
  return product_space(M, N, fp8_plan(M, N, K));
}

int rampde_fp8_matmul(int64_t M, int64_t N, int64_t K, const void* a_values, const void* a_scales, const void* b_values,
                      const void* b_scales, rampde_dtype c_type, int accumulate, void* C, int64_t ldc, void* workspace,
                      size_t workspace_bytes, void* hip_stream) {
  Fp8Args g{};
  Fp8Plan p;
  if (const int rc = check_product(M, N, K, a_values, a_scales, b_values, b_scales, c_type, accumulate, C, ldc, workspace, workspace_bytes, g, p))
    return rc;
  return by_type(c_type, [&](auto tag) { return multiply<decltype(tag), false>(g, p, (hipStream_t)hip_stream); });
}

int rampde_fp8_matmul_short(int64_t M, int64_t N, int64_t K, const void* a_values, const void* a_scales, const void* b_values,
                            const void* b_scales, rampde_dtype c_type, void* C, int64_t ldc, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  if (c_type == RAMPDE_F32) return RAMPDE_EINVAL;  // (it would hold places that the sums do not have)
  Fp8Args g{};
  Fp8Plan p;
  if (const int rc = check_product(M, N, K, a_values, a_scales, b_values, b_scales, c_type, 0, C, ldc, workspace, workspace_bytes, g, p)) return rc;
  return c_type == RAMPDE_F16 ? multiply<F16, true>(g, p, (hipStream_t)hip_stream) : multiply<BF16, true>(g, p, (hipStream_t)hip_stream);
}

}  // extern "C"
