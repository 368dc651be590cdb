// Dropout (rampde_dropout), and the end of a residual block fused with the head of the next one (rampde_join_fwd / _bwd):
//     y' = y + alpha scale s(gate) k (N(b) w_post),   x = N(y') w_pre,   N(v) = v / sqrt(mean(v^2) + eps).
// All of it is one pass over the rows: a row stays in the registers of the lanes that share it, its two sums of squares are
// folded across them, and what the forward pass keeps for the backward pass is the two reciprocal roots of a row.
// Backward, with n = N(b), m = N(y') and the row means <.>:
//     dv = dy' + r_pre (t - m <t m>),  t = dx w_pre;         dw_pre += sum_rows dx m
//     dn = dv alpha scale s k;   u = dn w_post;              db = r_post (u - n <u n>),   dw_post += sum_rows dn n
//     dscale += sum_rows dv alpha s k n w_post;              dgate = dv alpha scale k n w_post s (1 - s);    dy = dv
// Column sums are kept in registers over the rows of a workgroup, written as one copy per workgroup and folded in a fixed order.
//
// Memory bounds it: an element is 14 bytes forward (y, b, gate in, y', x out, with b, gate and x in 16 bits) and 22 backward (y', b,
// gate, dy', dx in, dy, db, dgate out).  Measured on 16384 x 2048 in bf16 with gate and dropout: forward 91 us (5.2 TB/s), backward 149 us
// (5.0 TB/s) and 5 us to fold the column sums; a plain copy of that size reaches 5.05 TB/s.  Columns in no multiple of eight cost
// accesses across cache lines, and draws of two blocks of the generator for eight elements: 16384 x 1001 47 us forward, 1024 columns 40.
// Beyond 8192 columns the backward pass has twice the columns in a lane and spills: 236 us (1.6 TB/s) at 1024 x 16384.  Few rows are
// bound by latency: 16 x 2048 4.7 us, 1003 x 1001 in f16 8 us forward and 11 + 5 us backward.
#include <algorithm>
#include <cmath>
#include "entry.hpp"
#include "element.hpp"
#include "philox.hpp"

namespace rampde {
namespace {

// ------------------------------------------------------------------ dropout
// Eight elements per lane, which one block of the generator covers (ten rounds of two 32 x 32 -> 64 bit products: 16 random bits per
// element are enough for p in steps of 2^-16).  Memory bounds it, 2 + 2 bytes per element in 16 bits: 67 million elements take
// 41 us (6.6 TB/s, part of it from the last-level cache); in fp32 160 million take 249 us (5.1 TB/s).
template <class T>
__global__ __launch_bounds__(256) void dropout_elements(const typename Elem<T>::S* x, typename Elem<T>::S* out, int64_t n, Mask m) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q * 8 < n; q += stride) {
    const int64_t e = q * 8;
    const int left = n - e < 8 ? (int)(n - e) : 8;
    float v[8], k[8];
    unpack8<T>(load8<T>(x + e, left), v);
    mask8(m, (uint64_t)e, k);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k[i] != 0.f ? v[i] * k[i] : 0.f;
    store8<T>(out + e, left, v);
  }
}

// ------------------------------------------------------------------ join
struct JoinArgs {
  const float* y;        // forward: y; backward: y'
  const void* b;
  const void* gate;
  const float* w_post;
  const float* scale;
  const float* w_pre;
  float* y_out;          // backward: dy
  void* x;               // backward: dx
  float* rstd;
  const float* dy_out;
  void* db;
  void* dgate;
  float* part;           // backward: [workgroups][3][cols]
  int64_t rows;
  int cols;
  float alpha, eps;
  Mask m;
  int64_t ld_b, ld_gate, ld_x;
};

// A row is shared by L lanes of a wavefront (narrow rows: fewer than 64) or by W wavefronts, 8 L NV columns each, of which a lane has
// eight neighbouring ones (NV times); a workgroup has R (64 / L) rows.  WHOLE: the number of columns is a multiple of eight.
//
// Sum over the lanes that share a row.  sh: W > 1, the workgroup's wavefronts; a kernel's sums take turns between two such arrays,
// so that one barrier a sum is enough (the readers of an array have passed the other sum's barrier when it is written again).
// Every thread of the workgroup must get here.
template <int W, int L>
__device__ inline float row_sum(float v, float* sh) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (W > 1) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) sh[w] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += sh[w / W * W + i];
  }
  return v;
}

// the 8 entries of a vector of parameters (ones where it is absent)
template <bool WHOLE>
__device__ inline void load_vector(const float* p, int c, int cols, float (&f)[8]) {
  if (p) {
    unpack8<F32>(load8<F32>(p + c, WHOLE ? 8 : cols - c), f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 1.f;
  }
}

template <bool WHOLE, int L>
__device__ inline void row_mask(const Mask& m, int64_t row, int cols, int c, float (&k)[8]) {
  if constexpr (WHOLE) mask8(m, (uint64_t)(row * cols + c), k);
  else mask8_any<L>(m, (uint64_t)(row * cols + c), cols <= 8 * (L - 1), k);
}

template <class T, int W, int L, int R, int NV, bool WHOLE>
__global__ __launch_bounds__(64 * W * R) void join_forward(JoinArgs g) {
  typedef typename Elem<T>::S S;
  __shared__ float sh[2][W * R];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % W, sub = wave / W, li = lane % L;
  constexpr int ROWS = R * (64 / L);
  const int c0 = w * 8 * L * NV + li * 8;
  const float inv = 1.f / (float)g.cols;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < g.rows; r0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = r0 + sub * (64 / L) + lane / L;
    const bool live = row < g.rows;
    Raw8<F32> yr[NV] = {};
    Raw8<T> br[NV] = {}, gr[NV] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + 8 * L * j;
      if (live && c < g.cols) {
        if (g.b) br[j] = load8<T>((const S*)g.b + row * g.ld_b + c, WHOLE ? 8 : g.cols - c);
        yr[j] = load8<F32>(g.y + row * g.cols + c, WHOLE ? 8 : g.cols - c);
        if (g.gate) gr[j] = load8<T>((const S*)g.gate + row * g.ld_gate + c, WHOLE ? 8 : g.cols - c);
      }
    }
    float y[NV][8], b[NV][8];
    float s1 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      unpack8<F32>(yr[j], y[j]);
      unpack8<T>(br[j], b[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s1 = fmaf(b[j][i], b[j][i], s1);
    }
    const float r_post = 1.f / sqrtf(fmaf(row_sum<W, L>(s1, sh[0]), inv, g.eps));
    float s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + 8 * L * j;
      if (g.b) {
        float wp[8], sc[8], k[8];
        if (g.m.drop) row_mask<WHOLE, L>(g.m, row, g.cols, c, k);  // (lanes past the row's end draw factors of other elements: not used)
        if (live && c < g.cols) {
          load_vector<WHOLE>(g.w_post, c, g.cols, wp);
          load_vector<WHOLE>(g.scale, c, g.cols, sc);
          if (g.gate) {
            float gt[8];
            unpack8<T>(gr[j], gt);
#pragma unroll
            for (int i = 0; i < 8; ++i) sc[i] *= logistic<T>(gt[i]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float f = g.m.drop ? g.alpha * sc[i] * k[i] : g.alpha * sc[i];
            y[j][i] = WHOLE || c + i < g.cols ? fmaf(f, b[j][i] * r_post * wp[i], y[j][i]) : 0.f;
          }
          store8<F32>(g.y_out + row * g.cols + c, WHOLE ? 8 : g.cols - c, y[j]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s2 = fmaf(y[j][i], y[j][i], s2);
    }
    const float r_pre = 1.f / sqrtf(fmaf(row_sum<W, L>(s2, sh[1]), inv, g.eps));
    if (g.rstd && live && w == 0 && li == 0) {
      g.rstd[row] = r_post;
      g.rstd[g.rows + row] = r_pre;
    }
    if (g.x && live) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = c0 + 8 * L * j;
        if (c < g.cols) {
          float wp[8];
          load_vector<WHOLE>(g.w_pre, c, g.cols, wp);
#pragma unroll
          for (int i = 0; i < 8; ++i) wp[i] *= y[j][i] * r_pre;
          store8<T>((S*)g.x + row * g.ld_x + c, WHOLE ? 8 : g.cols - c, wp);
        }
      }
    }
  }
}

template <class T, int W, int L, int R, int NV, bool WHOLE>
__global__ __launch_bounds__(64 * W * R, sizeof(typename Elem<T>::S) == 2 ? 4 : 1) void join_backward(JoinArgs g) {
  typedef typename Elem<T>::S S;
  __shared__ float sh[2][W * R];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % W, sub = wave / W, li = lane % L;
  constexpr int ROWS = R * (64 / L);
  const int c0 = w * 8 * L * NV + li * 8;
  const float inv = 1.f / (float)g.cols;
  float cs[3][NV][8];  // column sums: dw_post, dscale, dw_pre
#pragma unroll
  for (int q = 0; q < 3; ++q)
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[q][j][i] = 0.f;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < g.rows; r0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = r0 + sub * (64 / L) + lane / L;
    const bool live = row < g.rows;
    const float r_post = live && g.b ? g.rstd[row] : 0.f, r_pre = live && g.x ? g.rstd[g.rows + row] : 0.f;
    Raw8<F32> yr[NV] = {}, vr[NV] = {};
    Raw8<T> xr[NV] = {}, br[NV] = {}, gr[NV] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + 8 * L * j;
      if (live && c < g.cols) {
        if (g.x) {
          xr[j] = load8<T>((const S*)g.x + row * g.ld_x + c, WHOLE ? 8 : g.cols - c);
          yr[j] = load8<F32>(g.y + row * g.cols + c, WHOLE ? 8 : g.cols - c);
        }
        if (g.dy_out) vr[j] = load8<F32>(g.dy_out + row * g.cols + c, WHOLE ? 8 : g.cols - c);
        if (g.b) br[j] = load8<T>((const S*)g.b + row * g.ld_b + c, WHOLE ? 8 : g.cols - c);
        if (g.gate) gr[j] = load8<T>((const S*)g.gate + row * g.ld_gate + c, WHOLE ? 8 : g.cols - c);
      }
    }
    float dv[NV][8], m[NV][8];
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + 8 * L * j;
      float d[8], wq[8];
      unpack8<T>(xr[j], d);
      unpack8<F32>(yr[j], m[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) wq[i] = 0.f;
      if (g.x && c < g.cols) load_vector<WHOLE>(g.w_pre, c, g.cols, wq);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[j][i] *= r_pre;
        cs[2][j][i] = fmaf(d[i], m[j][i], cs[2][j][i]);
        dv[j][i] = d[i] * wq[i];
        s = fmaf(dv[j][i], m[j][i], s);
      }
    }
    s = row_sum<W, L>(s, sh[0]) * inv;
    float u[NV][8], nb[NV][8];
    float s1 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + 8 * L * j;
      float d[8], k[8];
      unpack8<F32>(vr[j], d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dv[j][i] = fmaf(r_pre, dv[j][i] - m[j][i] * s, d[i]);
        u[j][i] = 0.f;
      }
      unpack8<T>(br[j], nb[j]);
      if (g.b && g.m.drop) row_mask<WHOLE, L>(g.m, row, g.cols, c, k);
      if (live && c < g.cols) {
        store8<F32>(g.y_out + row * g.cols + c, WHOLE ? 8 : g.cols - c, dv[j]);
        if (g.b) {
          float wp[8], sc[8], gt[8], dg[8];
          load_vector<WHOLE>(g.w_post, c, g.cols, wp);
          load_vector<WHOLE>(g.scale, c, g.cols, sc);
          unpack8<T>(gr[j], gt);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const Gate v = gate_of<T>(gt[i]);
            const float gv = g.gate ? v.s : 1.f;
            nb[j][i] *= r_post;
            const float da = g.m.drop ? g.alpha * dv[j][i] * k[i] : g.alpha * dv[j][i];  // of s(gate) scale N(b) w_post
            const float dn = da * gv * sc[i];                                            // of N(b) w_post
            cs[0][j][i] = fmaf(dn, nb[j][i], cs[0][j][i]);
            cs[1][j][i] = fmaf(da * gv, nb[j][i] * wp[i], cs[1][j][i]);
            u[j][i] = dn * wp[i];
            dg[i] = u[j][i] * nb[j][i] * (fminf(v.e, 0x1p126f) * v.s);  // (1 - s; where e overflows s is 0, and so is u)
            s1 = fmaf(u[j][i], nb[j][i], s1);
          }
          if (g.dgate) store8<T>((S*)g.dgate + row * g.ld_gate + c, WHOLE ? 8 : g.cols - c, dg);
        }
      }
    }
    s1 = row_sum<W, L>(s1, sh[1]) * inv;
    if (g.b && live) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = c0 + 8 * L * j;
        if (c < g.cols) {
#pragma unroll
          for (int i = 0; i < 8; ++i) u[j][i] = r_post * (u[j][i] - nb[j][i] * s1);
          store8<T>((S*)g.db + row * g.ld_b + c, WHOLE ? 8 : g.cols - c, u[j]);
        }
      }
    }
  }
  // one copy of the column sums per workgroup: those of a wavefront's rows, then those of the wavefronts, are added in a fixed order
  if constexpr (L < 64) {
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int o = L; o < 64; o <<= 1) cs[q][j][i] += __shfl_xor(cs[q][j][i], o);
  }
  if constexpr (R > 1) {
    __shared__ float fold[R > 1 ? W : 1][NV][8][64];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      for (int from = 1; from < R; ++from) {
        __syncthreads();
        if (sub == from)
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) fold[w][j][i][lane] = cs[q][j][i];
        __syncthreads();
        if (sub == 0)
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[q][j][i] += fold[w][j][i][lane];
      }
    }
  }
  if (sub == 0 && lane < L)
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = c0 + 8 * L * j;
        if (c < g.cols) store8<F32>(g.part + ((int64_t)blockIdx.x * 3 + q) * g.cols + c, WHOLE ? 8 : g.cols - c, cs[q][j]);
      }
}

// grad = or += the copies' sum, in a fixed order.  grid (cols / 64, 3), 1024 threads = 16 phases x 64 columns
__global__ __launch_bounds__(1024) void join_fold(const float* part, int copies, int cols, int write, float* dw_post, float* dscale,
                                                  float* dw_pre) {
  float* out = blockIdx.y == 0 ? dw_post : blockIdx.y == 1 ? dscale : dw_pre;
  if (!out) return;
  const int lane = threadIdx.x & 63, ph = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int i = ph; i < copies; i += 16) s += part[((int64_t)i * 3 + blockIdx.y) * cols + c];
  }
  __shared__ float sh[16][64];
  sh[ph][lane] = s;
  __syncthreads();
  if (ph == 0 && c < cols) {
    for (int i = 1; i < 16; ++i) s += sh[i][lane];
    out[c] = write ? s : out[c] + s;
  }
}

Mask mask_of(double p, uint64_t seed, uint64_t offset) {
  Mask m;
  m.seed0 = (uint32_t)seed;
  m.seed1 = (uint32_t)(seed >> 32);
  m.offset = offset;
  m.drop = (uint32_t)std::lrint(p * 65536.0);
  m.scale = m.drop < 65536 ? 65536.f / (float)(65536 - m.drop) : 0.f;
  return m;
}

int check_join(const rampde_join* j, JoinArgs& g) {
  if (!j || j->rows < 1 || j->cols < 1 || !known_type(j->low)) return RAMPDE_EINVAL;
  g.alpha = (float)j->alpha;
  g.eps = (float)j->eps;
  if (!(j->p >= 0.0 && j->p <= 1.0) || !(g.eps > 0.f) || !std::isfinite(g.eps) || !std::isfinite(g.alpha)) return RAMPDE_EINVAL;  // (as fp32)
  if (j->cols > 16384) return RAMPDE_EUNSUPPORTED;
  const int64_t most = (int64_t)1 << 40;
  g.ld_b = j->ld_b ? j->ld_b : j->cols;
  g.ld_gate = j->ld_gate ? j->ld_gate : j->cols;
  g.ld_x = j->ld_x ? j->ld_x : j->cols;
  if (g.ld_b < j->cols || g.ld_gate < j->cols || g.ld_x < j->cols || g.ld_b > most || g.ld_gate > most || g.ld_x > most) return RAMPDE_EINVAL;
  if (j->rows > ((int64_t)1 << 46) / std::max({g.ld_b, g.ld_gate, g.ld_x})) return RAMPDE_EUNSUPPORTED;  // (offsets fit 64 bits)
  g.rows = j->rows;
  g.cols = (int)j->cols;
  g.m = mask_of(j->p, j->seed, j->offset);
  return RAMPDE_OK;
}

// Lanes and wavefronts of a row (8 columns per lane; beyond 8192 columns 16), rows of a workgroup, and workgroups of the backward pass,
// each of which leaves a copy of the column sums: two on a compute unit.  Rows of at most 64, 128 or 256 columns share a wavefront
// (65536 x 64, bf16: forward 13 us, with 16 lanes a row 16, with a wavefront 28; backward with its fold 27 and 34).  The forward pass
// has wavefronts for three quarters of a power of two too (4096 x 6000, bf16: 74 us, with 16 wavefronts 93; 8192 x 3000: 77 and 79); the
// backward pass gains nothing by them (138 and 138, 131 and 128 us).
int lanes_per_row(int64_t cols) { return cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64; }
int waves_per_row(int64_t cols, bool back) {
  for (const int w : {1, 2, 3, 4, 6, 8, 12})
    if (cols <= 512 * w && !(back && w % 3 == 0)) return w;
  return 16;
}
int rows_per_group(int64_t cols, bool back) { return std::max(1, (back ? 8 : 4) / waves_per_row(cols, back)) * (64 / lanes_per_row(cols)); }
int join_groups(int64_t rows, int64_t cols) {
  const int r = rows_per_group(cols, true);
  return (int)std::min<int64_t>((rows + r - 1) / r, 512);
}

template <bool BACK, class T, int W, int L, int NV>
int join_launch(const JoinArgs& g, bool whole, hipStream_t st) {
  constexpr int R = std::max(1, (BACK ? 8 : 4) / W);
  if constexpr (BACK) {
    const unsigned grid = (unsigned)join_groups(g.rows, g.cols);
    if (whole) join_backward<T, W, L, R, NV, true><<<grid, 64 * W * R, 0, st>>>(g);
    else join_backward<T, W, L, R, NV, false><<<grid, 64 * W * R, 0, st>>>(g);
  } else {
    const int rows = rows_per_group(g.cols, false);
    const unsigned grid = (unsigned)std::min<int64_t>((g.rows + rows - 1) / rows, 65536);
    if (whole) join_forward<T, W, L, R, NV, true><<<grid, 64 * W * R, 0, st>>>(g);
    else join_forward<T, W, L, R, NV, false><<<grid, 64 * W * R, 0, st>>>(g);
  }
  HIP_TRY(hipGetLastError());
  return RAMPDE_OK;
}

template <bool BACK, class T>
int join_by_cols(const JoinArgs& g, bool whole, hipStream_t st) {
  switch (lanes_per_row(g.cols)) {
    case 8: return join_launch<BACK, T, 1, 8, 1>(g, whole, st);
    case 16: return join_launch<BACK, T, 1, 16, 1>(g, whole, st);
    case 32: return join_launch<BACK, T, 1, 32, 1>(g, whole, st);
  }
  if constexpr (!BACK) {
    switch (waves_per_row(g.cols, false)) {
      case 3: return join_launch<BACK, T, 3, 64, 1>(g, whole, st);
      case 6: return join_launch<BACK, T, 6, 64, 1>(g, whole, st);
      case 12: return join_launch<BACK, T, 12, 64, 1>(g, whole, st);
    }
  }
  switch (waves_per_row(g.cols, BACK)) {
    case 1: return join_launch<BACK, T, 1, 64, 1>(g, whole, st);
    case 2: return join_launch<BACK, T, 2, 64, 1>(g, whole, st);
    case 4: return join_launch<BACK, T, 4, 64, 1>(g, whole, st);
    case 8: return join_launch<BACK, T, 8, 64, 1>(g, whole, st);
    default: return g.cols <= 8192 ? join_launch<BACK, T, 16, 64, 1>(g, whole, st) : join_launch<BACK, T, 16, 64, 2>(g, whole, st);
  }
}

template <bool BACK>
int join_by_type(rampde_dtype t, const JoinArgs& g, hipStream_t st) {
  const bool whole = g.cols % 8 == 0;
  return by_type(t, [&](auto tag) { return join_by_cols<BACK, decltype(tag)>(g, whole, st); });
}

}  // namespace
}  // namespace rampde

using namespace rampde;

extern "C" {

int rampde_dropout(rampde_dtype low, int64_t n, const void* x, double p, uint64_t seed, uint64_t offset, void* out, void* hip_stream) {
  if (!known_type(low) || n < 1 || !x || !out || !(p >= 0.0 && p <= 1.0)) return RAMPDE_EINVAL;
  const size_t e = type_size(low);
  if (!aligned_to(x, e) || !aligned_to(out, e)) return RAMPDE_EINVAL;
  if (n >= (int64_t)1 << 40) return RAMPDE_EUNSUPPORTED;
  const Mask m = mask_of(p, seed, offset);
  const int64_t all = (n + 2047) / 2048;
  const unsigned grid = (unsigned)(all < 4096 ? all : 4096);
  const hipStream_t st = (hipStream_t)hip_stream;
  return by_type(low, [&](auto tag) {
    typedef decltype(tag) T;
    typedef typename Elem<T>::S S;
    dropout_elements<T><<<grid, 256, 0, st>>>((const S*)x, (S*)out, n, m);
    HIP_TRY(hipGetLastError());
    return (int)RAMPDE_OK;
  });
}

size_t rampde_join_workspace_bytes(const rampde_join* j) {
  JoinArgs g{};
  if (check_join(j, g) != RAMPDE_OK) return 0;
  return ((size_t)join_groups(j->rows, j->cols) * 3 * j->cols * 4 + 255) & ~(size_t)255;
}

int rampde_join_fwd(const rampde_join* j, const float* y, const void* b, const void* gate, const float* w_post, const float* scale,
                    const float* w_pre, float* y_out, void* x, float* rstd, void* hip_stream) {
  JoinArgs g{};
  if (const int rc = check_join(j, g)) return rc;
  const size_t e = type_size(j->low);
  if (!y || (b ? !y_out : (y_out || gate)) || (!b && !x)) return RAMPDE_EINVAL;
  if (!aligned_to(y, 4) || !aligned_to(b, e) || !aligned_to(gate, e) || !aligned_to(w_post, 4) || !aligned_to(scale, 4) ||
      !aligned_to(w_pre, 4) || !aligned_to(y_out, 4) || !aligned_to(x, e) || !aligned_to(rstd, 4))
    return RAMPDE_EINVAL;
  g.y = y, g.b = b, g.gate = gate, g.w_post = w_post, g.scale = scale, g.w_pre = w_pre, g.y_out = y_out, g.x = x, g.rstd = rstd;
  return join_by_type<false>(j->low, g, (hipStream_t)hip_stream);
}

int rampde_join_bwd(const rampde_join* j, const float* y_out, const void* b, const void* gate, const float* w_post,
                    const float* scale, const float* w_pre, const float* rstd, const float* dy_out, const void* dx, float* dy,
                    void* db, void* dgate, float* dw_post, float* dscale, float* dw_pre, void* workspace, size_t workspace_bytes,
                    void* hip_stream) {
  JoinArgs g{};
  if (const int rc = check_join(j, g)) return rc;
  const size_t e = type_size(j->low);
  if (!y_out || !rstd || !dy || (b ? !db : (db || gate)) || (gate ? !dgate : dgate != nullptr)) return RAMPDE_EINVAL;
  if (!aligned_to(y_out, 4) || !aligned_to(b, e) || !aligned_to(gate, e) || !aligned_to(w_post, 4) || !aligned_to(scale, 4) ||
      !aligned_to(w_pre, 4) || !aligned_to(rstd, 4) || !aligned_to(dy_out, 4) || !aligned_to(dx, e) || !aligned_to(dy, 4) ||
      !aligned_to(db, e) || !aligned_to(dgate, e) || !aligned_to(dw_post, 4) || !aligned_to(dscale, 4) || !aligned_to(dw_pre, 4))
    return RAMPDE_EINVAL;
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < rampde_join_workspace_bytes(j)) return RAMPDE_EWORKSPACE;
  g.y = y_out, g.b = b, g.gate = gate, g.w_post = w_post, g.scale = scale, g.w_pre = w_pre, g.rstd = const_cast<float*>(rstd);
  g.dy_out = dy_out, g.x = const_cast<void*>(dx), g.y_out = dy, g.db = db, g.dgate = dgate, g.part = (float*)workspace;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (const int rc = join_by_type<true>(j->low, g, st)) return rc;
  if (dw_post || dscale || dw_pre) {
    // (without a branch, without x, the copies hold zeros: what is left unchanged, or zero)
    join_fold<<<dim3((unsigned)((g.cols + 63) / 64), 3), 1024, 0, st>>>(g.part, join_groups(g.rows, g.cols), g.cols, j->write_grads, dw_post,
                                                                        dscale, dw_pre);
    HIP_TRY(hipGetLastError());
  }
  return RAMPDE_OK;
}

}  // extern "C"
