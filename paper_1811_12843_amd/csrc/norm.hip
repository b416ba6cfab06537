// Root-mean-square norm with the residual's addition and its gradients
// (lipz_rms_norm, lipz_rms_norm_backward).
//
// A group of TPR lanes owns a row: it reads x and residual once, 8 elements
// per lane and access, keeps the row's fp32 sums h in registers, reduces the
// squares over the group, and writes h and y (or, for e4m3, reduces max |y|
// first).  The backward pass keeps h rstd and dy gamma of the row and, over all
// rows of the group, the columns' sums of dy h rstd; a block adds its groups'
// in LDS and a second kernel the blocks', each in a fixed order.
//
// TPR lanes with NV accesses each hold a row: up to 512 columns the fewest of 8 ..
// 64 lanes with one access, so that short rows share a wave; up to 2048 a wave with
// two or four; up to 8192 a block of 256 threads, then one of 1024, with two or
// four; rows over 32768 columns (16384 in the backward
// pass, which keeps more of a row) are read again for each of their passes
// instead.
//
// Bound by memory, each input read once: 16384 x 4096 bf16 with residual 94 us
// (5.7 TB/s; a large copy runs at 4.8), gradients of 8192 x 8192 bf16 108 us (5.0
// TB/s, 6 us of it the columns' sums); one row of 4096 to e4m3 6.6 us, a launch.
#include "block.h"

namespace lipz {
namespace {

constexpr int kMaxNormRows = 1 << 30;  // a row index and a grid's stride (2^17 at most) stay below 2^31

struct NormArgs {
  const void *x, *r;
  void *h, *y;
  int64_t x_ld, x_cell, r_ld, r_cell, h_ld, h_cell, y_ld, y_cell, gamma_cell;
  const float* gamma;
  float *rstd, *scale;
  int rows, cols;
  float eps;
};

struct NormBwdArgs {
  const void *h, *dy, *dh;
  void* dx;
  int64_t h_ld, h_cell, dy_ld, dy_cell, dh_ld, dh_cell, dx_ld, dx_cell, gamma_cell;
  const float *gamma, *rstd;
  float* part;  // [cells][gridDim.x][cols], NULL without dgamma
  int rows, cols;
};

template <int TPR>
struct Group {
  static constexpr int NT = TPR < 256 ? 256 : TPR;  // threads of a block
  static constexpr int N = NT / TPR;                // groups of a block
  // Reductions of a block alternate between two rows of `red`, so that one
  // barrier per reduction is enough.
  template <class Op>
  static __device__ __forceinline__ float all(float v, float (*red)[16], int& turn, Op op) {
#pragma unroll
    for (int s = 1; s < (TPR < 64 ? TPR : 64); s <<= 1) v = op(v, __shfl_xor(v, s, 64));
    if (TPR > 64) {
      float* to = red[turn & 1];
      ++turn;
      if ((threadIdx.x & 63) == 0) to[threadIdx.x >> 6] = v;
      __syncthreads();
      v = to[0];
#pragma unroll
      for (int w = 1; w < TPR / 64; ++w) v = op(v, to[w]);
    }
    return v;
  }
};

struct Add {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct MaxNan {
  __device__ __forceinline__ float operator()(float a, float b) const { return max_nan(a, b); }
};

// h of 8 columns from col on (zeros past the row)
template <class T>
__device__ __forceinline__ f32x8 residual_sum(const T* x, const T* r, int col, int cols) {
  f32x8 h = load8(x + col, cols - col);
  if (r) {
    const f32x8 b = load8(r + col, cols - col);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] += b[e];
  }
  return h;
}

template <class T, bool FP8>
__device__ __forceinline__ void put_y(void* y, int64_t at, int n, f32x8 v, float scale) {
  if (FP8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] / scale;
    store8_fp8((uint8_t*)y + at, n, v);
  } else {
    store8((T*)y + at, n, v);
  }
}

template <class T, bool FP8, int TPR, int NV>
__global__ __launch_bounds__(Group<TPR>::NT) void rms_norm_kernel(const NormArgs P) {
  using G = Group<TPR>;
  __shared__ float red[2][16];
  int turn = 0;
  const int c = blockIdx.y, t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  f32x8 gm[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = 8 * (v * TPR + t);
    gm[v] = col < P.cols ? row8(P.gamma + c * P.gamma_cell, col, P.cols) : f32x8{};
  }
  for (int row = blockIdx.x * G::N + grp; row < P.rows; row += gridDim.x * G::N) {
    const T* x = (const T*)P.x + c * P.x_cell + row * P.x_ld;
    const T* r = P.r ? (const T*)P.r + c * P.r_cell + row * P.r_ld : nullptr;
    f32x8 h[NV];
    typename Vec8<T>::type a[NV], b[NV];
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      a[v] = col < P.cols ? row8_raw(x, col, P.cols) : typename Vec8<T>::type{};
      if (r) b[v] = col < P.cols ? row8_raw(r, col, P.cols) : typename Vec8<T>::type{};
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      h[v] = widen<T>(row8_in_place<T>(a[v], col, P.cols));
      if (r) {
        const f32x8 w = widen<T>(row8_in_place<T>(b[v], col, P.cols));
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] += w[e];
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(h[v][e], h[v][e], ss);
    ss = G::all(ss, red, turn, Add());
    const float rstd = 1.f / sqrtf(ss / (float)P.cols + P.eps);
    if (P.h) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = 8 * (v * TPR + t);
        if (col < P.cols) store8((T*)P.h + c * P.h_cell + row * P.h_ld + col, P.cols - col, h[v]);
      }
    }
    float m = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[v][e] = h[v][e] * rstd * gm[v][e];
        if (FP8) m = max_nan(m, __builtin_fabsf(h[v][e]));
      }
    float scale = 1.f;
    if (FP8) scale = fp8_scale(G::all(m, red, turn, MaxNan()));
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      if (col < P.cols) put_y<T, FP8>(P.y, c * P.y_cell + row * P.y_ld + col, P.cols - col, h[v], scale);
    }
    if (t == 0) {
      if (P.rstd) P.rstd[(int64_t)c * P.rows + row] = rstd;
      if (FP8) P.scale[(int64_t)c * P.rows + row] = scale;
    }
  }
}

// Rows that registers do not hold: read again for y (and once more for its
// largest magnitude).  h is written in the last pass, after every read of the
// element, so that it may be x or residual.
template <class T, bool FP8>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(const NormArgs P) {
  using G = Group<1024>;
  __shared__ float red[2][16];
  int turn = 0;
  const int c = blockIdx.y, t = threadIdx.x;
  const float* gamma = P.gamma + c * P.gamma_cell;
  for (int row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* x = (const T*)P.x + c * P.x_cell + row * P.x_ld;
    const T* r = P.r ? (const T*)P.r + c * P.r_cell + row * P.r_ld : nullptr;
    float ss = 0.f;
    for (int col = 8 * t; col < P.cols; col += 8192) {
      const f32x8 h = residual_sum(x, r, col, P.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(h[e], h[e], ss);
    }
    ss = G::all(ss, red, turn, Add());
    const float rstd = 1.f / sqrtf(ss / (float)P.cols + P.eps);
    float scale = 1.f;
    if (FP8) {
      float m = 0.f;
      for (int col = 8 * t; col < P.cols; col += 8192) {
        const f32x8 h = residual_sum(x, r, col, P.cols), g = load8(gamma + col, P.cols - col);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max_nan(m, __builtin_fabsf(h[e] * rstd * g[e]));
      }
      scale = fp8_scale(G::all(m, red, turn, MaxNan()));
    }
    for (int col = 8 * t; col < P.cols; col += 8192) {
      const int n = P.cols - col;
      f32x8 h = residual_sum(x, r, col, P.cols);
      const f32x8 g = load8(gamma + col, n);
      if (P.h) store8((T*)P.h + c * P.h_cell + row * P.h_ld + col, n, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = h[e] * rstd * g[e];
      put_y<T, FP8>(P.y, c * P.y_cell + row * P.y_ld + col, n, h, scale);
    }
    if (t == 0) {
      if (P.rstd) P.rstd[(int64_t)c * P.rows + row] = rstd;
      if (FP8) P.scale[(int64_t)c * P.rows + row] = scale;
    }
  }
}

template <class T, int TPR, int NV>
__global__ __launch_bounds__(Group<TPR>::NT) void rms_norm_bwd_kernel(const NormBwdArgs P) {
  using G = Group<TPR>;
  __shared__ float red[2][16];
  int turn = 0;
  const int c = blockIdx.y, t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  f32x8 gm[NV], dg[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = 8 * (v * TPR + t);
    gm[v] = col < P.cols ? row8(P.gamma + c * P.gamma_cell, col, P.cols) : f32x8{};
    dg[v] = f32x8{};
  }
  for (int row = blockIdx.x * G::N + grp; row < P.rows; row += gridDim.x * G::N) {
    const T* hp = (const T*)P.h + c * P.h_cell + row * P.h_ld;
    const T* yp = (const T*)P.dy + c * P.dy_cell + row * P.dy_ld;
    const T* rp = P.dh ? (const T*)P.dh + c * P.dh_cell + row * P.dh_ld : nullptr;
    const float rstd = as_global(P.rstd)[(int64_t)c * P.rows + row];
    typename Vec8<T>::type h[NV], dy[NV], dh[NV];  // converted twice rather than held in fp32
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      h[v] = col < P.cols ? row8_raw(hp, col, P.cols) : typename Vec8<T>::type{};
      dy[v] = col < P.cols ? row8_raw(yp, col, P.cols) : typename Vec8<T>::type{};
      dh[v] = col < P.cols && rp ? row8_raw(rp, col, P.cols) : typename Vec8<T>::type{};
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      h[v] = row8_in_place<T>(h[v], col, P.cols);
      dy[v] = row8_in_place<T>(dy[v], col, P.cols);
      dh[v] = row8_in_place<T>(dh[v], col, P.cols);
      const f32x8 x = widen<T>(h[v]), d = widen<T>(dy[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = x[e] * rstd;
        dg[v][e] = fmaf(d[e], xh, dg[v][e]);
        s = fmaf(d[e] * gm[v][e], xh, s);
      }
    }
    const float mean = G::all(s, red, turn, Add()) / (float)P.cols;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      forget(h[v]);
      forget(dy[v]);
      const f32x8 x = widen<T>(h[v]), d = widen<T>(dy[v]), r = widen<T>(dh[v]);
      f32x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(rstd, fmaf(-(x[e] * rstd), mean, d[e] * gm[v][e]), r[e]);
      if (col < P.cols) store8((T*)P.dx + c * P.dx_cell + row * P.dx_ld + col, P.cols - col, o);
    }
  }
  if (!P.part) return;
  float* part = P.part + ((int64_t)c * gridDim.x + blockIdx.x) * P.cols;
  if (G::N == 1) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = 8 * (v * TPR + t);
      if (col < P.cols) store8(part + col, P.cols - col, dg[v]);
    }
  } else {
    constexpr int W = 8 * TPR * NV;
    __shared__ float sums[G::N > 1 ? G::N : 1][G::N > 1 ? W : 1];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[grp][8 * (v * TPR + t) + e] = dg[v][e];
    __syncthreads();
    for (int col = threadIdx.x; col < P.cols; col += G::NT) {
      float s = 0.f;
#pragma unroll
      for (int q = 0; q < G::N; ++q) s += sums[q][col];
      part[col] = s;
    }
  }
}

// Long rows: the block's column sums live in its row of `part`.
template <class T>
__global__ __launch_bounds__(1024) void rms_norm_bwd_long_kernel(const NormBwdArgs P) {
  using G = Group<1024>;
  __shared__ float red[2][16];
  int turn = 0;
  const int c = blockIdx.y, t = threadIdx.x;
  const float* gamma = P.gamma + c * P.gamma_cell;
  float* part = P.part ? P.part + ((int64_t)c * gridDim.x + blockIdx.x) * P.cols : nullptr;
  if (part)
    for (int col = 8 * t; col < P.cols; col += 8192) store8(part + col, P.cols - col, f32x8{});
  for (int row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* hp = (const T*)P.h + c * P.h_cell + row * P.h_ld;
    const T* yp = (const T*)P.dy + c * P.dy_cell + row * P.dy_ld;
    const T* rp = P.dh ? (const T*)P.dh + c * P.dh_cell + row * P.dh_ld : nullptr;
    const float rstd = as_global(P.rstd)[(int64_t)c * P.rows + row];
    float s = 0.f;
    for (int col = 8 * t; col < P.cols; col += 8192) {
      const f32x8 h = load8(hp + col, P.cols - col), d = load8(yp + col, P.cols - col),
                  g = load8(gamma + col, P.cols - col);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(d[e] * g[e], h[e] * rstd, s);
    }
    const float mean = G::all(s, red, turn, Add()) / (float)P.cols;
    for (int col = 8 * t; col < P.cols; col += 8192) {
      const int n = P.cols - col;
      const f32x8 h = load8(hp + col, n), d = load8(yp + col, n), g = load8(gamma + col, n);
      f32x8 o = rp ? load8(rp + col, n) : f32x8{};
      f32x8 q = part ? load8(part + col, n) : f32x8{};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = h[e] * rstd;
        q[e] = fmaf(d[e], xh, q[e]);
        o[e] = fmaf(rstd, fmaf(-xh, mean, d[e] * g[e]), o[e]);
      }
      if (part) store8(part + col, n, q);
      store8((T*)P.dx + c * P.dx_cell + row * P.dx_ld + col, n, o);
    }
  }
}

}  // namespace

// out[c][col] = sum over the n rows of part[c]: 16 columns a block, 16 threads a
// column, thread g the rows g, g + 16, .. (eight in flight); then theirs in order.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* part, int n, int cols, float* out, int64_t out_cell) {
  __shared__ float sums[16][16 + 1];
  const int lane = threadIdx.x & 15, g = threadIdx.x >> 4, col = blockIdx.x * 16 + lane, c = blockIdx.y;
  const LIPZ_GLOBAL float* p = as_global(part) + (int64_t)c * n * cols + col;
  float s = 0.f;
  if (col < cols) {
    int i = g;
    for (; i + 112 < n; i += 128) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = p[(int64_t)(i + 16 * u) * cols];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; i < n; i += 16) s += p[(int64_t)i * cols];
  }
  sums[g][lane] = s;
  __syncthreads();
  if (g || col >= cols) return;
#pragma unroll
  for (int q = 1; q < 16; ++q) s += sums[q][lane];
  as_global(out)[c * out_cell + col] = s;
}

hipError_t launch_sum_parts(const float* part, int n, int cols, int cells, float* out, int64_t out_cell, hipStream_t s) {
  sum_parts_kernel<<<dim3((cols + 15) / 16, cells), 256, 0, s>>>(part, n, cols, out, out_cell);
  return hipGetLastError();
}

namespace {

// Threads per row and accesses per lane for rows of `cols`; tpr = 0: rows
// longer than `most`, which registers do not hold.
constexpr int kFwdMost = 32768, kBwdMost = 16384;
void row_shape(int cols, int most, int& tpr, int& nv) {
  const int v = (cols + 7) / 8;
  if (v <= 64) {
    tpr = v <= 8 ? 8 : v <= 16 ? 16 : v <= 32 ? 32 : 64;
    nv = 1;
  } else if (v <= 256) {
    tpr = 64;
    nv = v <= 128 ? 2 : 4;
  } else if (v <= 1024) {
    tpr = 256;
    nv = v <= 512 ? 2 : 4;
  } else if (cols <= most) {
    tpr = 1024;
    nv = v <= 2048 ? 2 : 4;
  } else {
    tpr = 0;
    nv = 0;
  }
}
int groups_of(int tpr) { return tpr && tpr < 256 ? 256 / tpr : 1; }

// Blocks per cell, of `most` over all cells, no more than there are rows for.
// Forward, a row per block up to 16384 blocks for rows over 2048 columns:
// rows then start as others end (16384 x 4096 bf16 94 us; 4096 blocks 99, 2048
// 105); 4096 for shorter ones, which share a block (200000 x 64 bf16 19.1 us;
// 16384 blocks 20.6, 2048 19.6); 512 for blocks of 1024 threads, two to a compute
// unit (2048 x 32768 bf16 108 us, 2048 blocks 115).  Backward 512: each adds a row
// to the columns' partial sums.
int norm_blocks(int rows, int cells, int tpr, int most) {
  const int per = groups_of(tpr);
  const int want = (most + cells - 1) / cells, have = (rows + per - 1) / per;
  return have < want ? have : want;
}
int fwd_blocks(int rows, int cells, int tpr) { return norm_blocks(rows, cells, tpr, tpr == 0 || tpr == 1024 ? 512 : tpr == 256 ? 16384 : 4096); }
int bwd_blocks(int rows, int cells, int tpr) { return norm_blocks(rows, cells, tpr, 512); }

template <class F>
void for_shape(int tpr, int nv, F f) {
#define LIPZ_SHAPE(T, N) \
  if (tpr == T && nv == N) f(std::integral_constant<int, T>(), std::integral_constant<int, N>());
  LIPZ_SHAPE(8, 1)
  LIPZ_SHAPE(16, 1)
  LIPZ_SHAPE(32, 1)
  LIPZ_SHAPE(64, 1)
  LIPZ_SHAPE(64, 2)
  LIPZ_SHAPE(64, 4)
  LIPZ_SHAPE(256, 2)
  LIPZ_SHAPE(256, 4)
  LIPZ_SHAPE(1024, 2)
  LIPZ_SHAPE(1024, 4)
#undef LIPZ_SHAPE
}

template <class T, bool FP8>
void launch_norm(const NormArgs& P, int cells, hipStream_t s) {
  int tpr, nv;
  row_shape(P.cols, kFwdMost, tpr, nv);
  const dim3 grid(fwd_blocks(P.rows, cells, tpr), cells);
  if (!tpr) rms_norm_long_kernel<T, FP8><<<grid, 1024, 0, s>>>(P);
  for_shape(tpr, nv, [&](auto t, auto n) {
    rms_norm_kernel<T, FP8, t.value, n.value><<<grid, Group<t.value>::NT, 0, s>>>(P);
  });
}

template <class T>
void launch_norm_bwd(const NormBwdArgs& P, int cells, int blocks, hipStream_t s) {
  int tpr, nv;
  row_shape(P.cols, kBwdMost, tpr, nv);
  const dim3 grid(blocks, cells);
  if (!tpr) rms_norm_bwd_long_kernel<T><<<grid, 1024, 0, s>>>(P);
  for_shape(tpr, nv, [&](auto t, auto n) {
    if constexpr (8 * t.value * n.value <= kBwdMost)
      rms_norm_bwd_kernel<T, t.value, n.value><<<grid, Group<t.value>::NT, 0, s>>>(P);
  });
}

lipz_status check_norm(const lipz_rms_norm_args* a) {
  if (!a || a->abi_version != LIPZ_ABI_VERSION) return LIPZ_E_INVAL;
  if (!valid_float(a->dtype) || (a->y_dtype != a->dtype && a->y_dtype != LIPZ_FP8)) return LIPZ_E_INVAL;
  if (a->cells < 1 || a->rows < 0 || a->cols < 1 || !(a->eps > 0.f) || !(a->eps < __builtin_inff())) return LIPZ_E_INVAL;
  if (a->cells > kMaxCells || a->rows > kMaxNormRows || a->cols > kMaxWide) return LIPZ_E_UNSUPPORTED;
  if (!a->gamma || (a->rows && (!a->x.p || !a->y.p || (a->y_dtype == LIPZ_FP8 && !a->y_scale)))) return LIPZ_E_INVAL;
  lipz_status st;
  if ((st = check_mat(a->x, a->cells, a->rows, a->cols, a->dtype, false))) return st;
  if (a->residual.p && (st = check_mat(a->residual, a->cells, a->rows, a->cols, a->dtype, false))) return st;
  if (a->h.p && (st = check_mat(a->h, a->cells, a->rows, a->cols, a->dtype, true))) return st;
  if ((st = check_mat(a->y, a->cells, a->rows, a->cols, a->y_dtype, true))) return st;
  if ((st = check_vec(a->gamma, a->gamma_cell, a->cells, a->cols, false))) return st;
  if (((uintptr_t)a->rstd | (uintptr_t)a->y_scale) % 4) return LIPZ_E_INVAL;
  return LIPZ_OK;
}

lipz_status check_norm_bwd(const lipz_rms_norm_backward_args* a) {
  if (!a || a->abi_version != LIPZ_ABI_VERSION || !valid_float(a->dtype)) return LIPZ_E_INVAL;
  if (a->cells < 1 || a->rows < 0 || a->cols < 1) return LIPZ_E_INVAL;
  if (a->cells > kMaxCells || a->rows > kMaxNormRows || a->cols > kMaxWide) return LIPZ_E_UNSUPPORTED;
  if (!a->gamma || (a->rows && (!a->h.p || !a->dy.p || !a->dx.p || !a->rstd)) || (uintptr_t)a->rstd % 4) return LIPZ_E_INVAL;
  lipz_status st;
  if ((st = check_mat(a->h, a->cells, a->rows, a->cols, a->dtype, false))) return st;
  if ((st = check_mat(a->dy, a->cells, a->rows, a->cols, a->dtype, false))) return st;
  if (a->dh.p && (st = check_mat(a->dh, a->cells, a->rows, a->cols, a->dtype, false))) return st;
  if ((st = check_mat(a->dx, a->cells, a->rows, a->cols, a->dtype, true))) return st;
  if ((st = check_vec(a->gamma, a->gamma_cell, a->cells, a->cols, false))) return st;
  if (a->dgamma && (st = check_vec(a->dgamma, a->dgamma_cell, a->cells, a->cols, true))) return st;
  return LIPZ_OK;
}

}  // namespace
}  // namespace lipz

using namespace lipz;

extern "C" {

size_t lipz_rms_norm_workspace_bytes(const lipz_rms_norm_args* a) { return check_norm(a) ? 0 : 256; }

lipz_status lipz_rms_norm(const lipz_rms_norm_args* a, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  lipz_status st = check_norm(a);
  if (st) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, 256))) return st;
  if (!a->rows) return LIPZ_OK;
  NormArgs P{};
  P.x = a->x.p, P.x_ld = a->x.ld, P.x_cell = a->x.cell;
  P.r = a->residual.p, P.r_ld = a->residual.ld, P.r_cell = a->residual.cell;
  P.h = a->h.p, P.h_ld = a->h.ld, P.h_cell = a->h.cell;
  P.y = a->y.p, P.y_ld = a->y.ld, P.y_cell = a->y.cell;
  P.gamma = a->gamma, P.gamma_cell = a->gamma_cell, P.rstd = a->rstd, P.scale = a->y_scale;
  P.rows = a->rows, P.cols = a->cols, P.eps = a->eps;
  hipStream_t s = (hipStream_t)hip_stream;
  const bool q = a->y_dtype == LIPZ_FP8;
  if (a->dtype == LIPZ_F32) q ? launch_norm<float, true>(P, a->cells, s) : launch_norm<float, false>(P, a->cells, s);
  else if (a->dtype == LIPZ_BF16) q ? launch_norm<__bf16, true>(P, a->cells, s) : launch_norm<__bf16, false>(P, a->cells, s);
  else q ? launch_norm<_Float16, true>(P, a->cells, s) : launch_norm<_Float16, false>(P, a->cells, s);
  return launched();
}

size_t lipz_rms_norm_backward_workspace_bytes(const lipz_rms_norm_backward_args* a) {
  if (check_norm_bwd(a)) return 0;
  int tpr, nv;
  row_shape(a->cols, kBwdMost, tpr, nv);
  const size_t blocks = a->rows ? (size_t)bwd_blocks(a->rows, a->cells, tpr) : 0;
  return 256 + (a->dgamma ? (4 * blocks * a->cells * a->cols + 255) / 256 * 256 : 0);
}

lipz_status lipz_rms_norm_backward(const lipz_rms_norm_backward_args* a, void* d_workspace, size_t workspace_bytes,
                                   void* hip_stream) {
  lipz_status st = check_norm_bwd(a);
  if (st) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, lipz_rms_norm_backward_workspace_bytes(a)))) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  int tpr, nv, blocks = 0;
  if (a->rows) {
    row_shape(a->cols, kBwdMost, tpr, nv);
    blocks = bwd_blocks(a->rows, a->cells, tpr);
    NormBwdArgs P{};
    P.h = a->h.p, P.h_ld = a->h.ld, P.h_cell = a->h.cell;
    P.dy = a->dy.p, P.dy_ld = a->dy.ld, P.dy_cell = a->dy.cell;
    P.dh = a->dh.p, P.dh_ld = a->dh.ld, P.dh_cell = a->dh.cell;
    P.dx = a->dx.p, P.dx_ld = a->dx.ld, P.dx_cell = a->dx.cell;
    P.gamma = a->gamma, P.gamma_cell = a->gamma_cell, P.rstd = a->rstd;
    P.part = a->dgamma ? (float*)d_workspace : nullptr;
    P.rows = a->rows, P.cols = a->cols;
    if (a->dtype == LIPZ_F32) launch_norm_bwd<float>(P, a->cells, blocks, s);
    else if (a->dtype == LIPZ_BF16) launch_norm_bwd<__bf16>(P, a->cells, blocks, s);
    else launch_norm_bwd<_Float16>(P, a->cells, blocks, s);
    if ((st = launched())) return st;
  }
  if (!a->dgamma) return LIPZ_OK;
  return launch_sum_parts((const float*)d_workspace, blocks, a->cols, a->cells, a->dgamma, a->dgamma_cell, s) == hipSuccess
             ? LIPZ_OK
             : LIPZ_E_HIP;
}

}  // extern "C"
