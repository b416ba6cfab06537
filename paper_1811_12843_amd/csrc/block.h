// Shared by the residual-block operators (norm.hip, linear.hip, linear_fp8.hip):
// element types, wide loads and stores at any alignment, activations, and the
// host's checks of matrices.
#pragma once

#include <type_traits>

#include "lipz_internal.h"

namespace lipz {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// ---- element types ----
// __bf16 and _Float16 convert from fp32 with one rounding to nearest even.

template <class T>
struct Vec8;
template <>
struct Vec8<float> {
  typedef float type __attribute__((ext_vector_type(8)));
};
template <>
struct Vec8<__bf16> {
  typedef __bf16 type __attribute__((ext_vector_type(8)));
};
template <>
struct Vec8<_Float16> {
  typedef _Float16 type __attribute__((ext_vector_type(8)));
};

// Eight elements in a row at the alignment of one: the hardware takes wide
// global accesses at any address; 16-byte aligned ones run faster.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight {
  typename Vec8<T>::type v;
};

// Elements 0 .. min(n, 8) - 1 at p as fp32, the rest 0.
template <class T>
__device__ __forceinline__ f32x8 load8(const T* p, int n) {
  if (n >= 8) return __builtin_convertvector(reinterpret_cast<const LIPZ_GLOBAL Eight<T>*>((const LIPZ_GLOBAL T*)p)->v, f32x8);
  f32x8 r = {};
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) r[e] = (float)as_global(p)[e];
  return r;
}
// Hides from the compiler what a raw eight holds, so that it converts it again
// instead of keeping the fp32 values in registers.
template <class V>
__device__ __forceinline__ void forget(V& v) {
  if constexpr (sizeof(V) == 16) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
    asm volatile("" : "+v"(w));
    v = __builtin_bit_cast(V, w);
  }
}

// Elements as load8 takes them, not yet converted.
template <class T>
__device__ __forceinline__ typename Vec8<T>::type load8_raw(const T* p, int n) {
  if (n >= 8) return reinterpret_cast<const LIPZ_GLOBAL Eight<T>*>((const LIPZ_GLOBAL T*)p)->v;
  typename Vec8<T>::type r = {};
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) r[e] = as_global(p)[e];
  return r;
}
template <class T>
__device__ __forceinline__ f32x8 widen(typename Vec8<T>::type v) {
  return __builtin_convertvector(v, f32x8);
}
// Eight elements of a row from column col on (a multiple of 8) in two steps, so
// that a row's end costs no branch before its loads: row8_raw loads the last
// eight columns where fewer than eight are left (one at a time if the row has
// fewer), and row8_in_place moves them to their places, zeros past the row.
// One wide load where load8_raw takes up to seven that wait for each other.
template <class T>
__device__ __forceinline__ typename Vec8<T>::type row8_raw(const T* row, int col, int cols) {
  if (cols < 8) return load8_raw(row + col, cols - col);
  const LIPZ_GLOBAL T* p = (const LIPZ_GLOBAL T*)row + (col < cols - 8 ? col : cols - 8);
  return reinterpret_cast<const LIPZ_GLOBAL Eight<T>*>(p)->v;
}
template <class T>
__device__ __forceinline__ typename Vec8<T>::type row8_in_place(typename Vec8<T>::type v, int col, int cols) {
  using Raw = typename Vec8<T>::type;
  const int by = col - (cols - 8);
  if (cols < 8 || by <= 0) return v;
  if (by >= 8) return Raw{};
  const Raw none = {};
  if (by & 4) v = __builtin_shufflevector(v, none, 4, 5, 6, 7, 8, 8, 8, 8);
  if (by & 2) v = __builtin_shufflevector(v, none, 2, 3, 4, 5, 6, 7, 8, 8);
  if (by & 1) v = __builtin_shufflevector(v, none, 1, 2, 3, 4, 5, 6, 7, 8);
  return v;
}
template <class T>
__device__ __forceinline__ typename Vec8<T>::type row8(const T* row, int col, int cols) {
  return row8_in_place<T>(row8_raw(row, col, cols), col, cols);
}
template <class T>
__device__ __forceinline__ void store8(T* p, int n, f32x8 v) {
  const typename Vec8<T>::type w = __builtin_convertvector(v, typename Vec8<T>::type);
  if (n >= 8) {
    reinterpret_cast<LIPZ_GLOBAL Eight<T>*>((LIPZ_GLOBAL T*)p)->v = w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) as_global(p)[e] = w[e];
}

// e4m3: NaN stays NaN; callers scale so that nothing exceeds 448 by more than a rounding.
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
struct __attribute__((packed, aligned(1))) EightBytes {
  u32x2 v;
};
__device__ __forceinline__ u32x2 to_fp8(f32x8 v) {
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
  return u32x2{(unsigned)lo, (unsigned)hi};
}
__device__ __forceinline__ void store8_fp8(uint8_t* p, int n, f32x8 v) {
  const u32x2 w = to_fp8(v);
  if (n >= 8) {
    reinterpret_cast<LIPZ_GLOBAL EightBytes*>((LIPZ_GLOBAL uint8_t*)p)->v = w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) as_global(p)[e] = (uint8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
}

constexpr float kFp8Max = 448.f;
constexpr float kFp8MinScale = 1.17549435e-38f;  // 2^-126: its reciprocal and the quotients by it are finite

// max that keeps a NaN of either side
__device__ __forceinline__ float max_nan(float a, float b) { return (a > b || a != a) ? a : b; }
// The scale of a row of largest magnitude m >= 0, infinite or NaN: NaN for the
// last two.  m times the fp32 reciprocal, as torch divides a tensor by a number, so
// that values quantised there agree to the bit; m / scale may then be 448 and one
// unit in fp32's last place, which still rounds to 448.
__device__ __forceinline__ float fp8_scale(float m) {
  const float s = m * (1.f / kFp8Max);
  return s < __builtin_inff() ? (s < kFp8MinScale ? kFp8MinScale : s) : __builtin_nanf("");
}

// ---- activations: z -> act(z), and act'(z) ----
// FAST: for outputs that are rounded to 16 bits.  erfc as below, exponentials and
// reciprocals of the hardware's 1 ulp; else the library's functions.  Neither takes
// a small value as the difference of large ones: GELU and the slopes keep their
// relative accuracy down to the smallest normal numbers (but for e^(-z^2 / 2)'s own
// z^2 2^-23, and where a slope passes through 0).

constexpr float kInvSqrt2 = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;

template <bool FAST>
__device__ __forceinline__ float exp_of(float x) {
  return FAST ? __builtin_amdgcn_exp2f(x * 1.44269504088896341f) : expf(x);
}
template <bool FAST>
__device__ __forceinline__ float recip(float x) {
  return FAST ? __builtin_amdgcn_rcpf(x) : 1.f / x;
}
// Phi(z); with FAST e must be e^(-z^2 / 2)
template <bool FAST>
__device__ __forceinline__ float normal_cdf(float z, float e) {
  if (!FAST) return 0.5f * erfcf(-z * kInvSqrt2);
  // erfc(x) e^(x^2), 0 <= x <= 12, as a polynomial of t = 1 / (1 + 0.376 x) without a
  // constant term: a least-squares fit of the ratio, weighted until its largest
  // errors are alike, 8.3e-7 (of Phi(-|z|) itself, wherever z lies)
  const float x = __builtin_fabsf(z) * kInvSqrt2;
  const float t = recip<true>(fmaf(0.376f, x, 1.f));
  float p = fmaf(-0.13225922f, t, 0.37415940f);
  p = fmaf(p, t, -0.11272450f);
  p = fmaf(p, t, 0.27244622f);
  p = fmaf(p, t, 0.17082962f);
  p = fmaf(p, t, 0.21559894f);
  p = fmaf(p, t, 0.21194951f);
  const float q = 0.5f * p * t * e;  // Phi(-|z|)
  return z < 0.f ? q : 1.f - q;
}
template <bool FAST>
__device__ __forceinline__ float tanh_of(float z) {
  if (!FAST) return tanhf(z);
  const float z2 = z * z;
  const float small = z * fmaf(z2, fmaf(z2, fmaf(z2, -0.05396825397f, 0.13333333333f), -0.33333333333f), 1.f);
  const float big = fmaf(-2.f, recip<true>(1.f + exp_of<true>(2.f * z)), 1.f);
  return z2 < 0.0625f ? small : big;
}

// GELU, SiLU and their slopes at infinite z are their limits, not 0 times infinity: z
// goes no lower than where e^z and Phi(z) are 0 in fp32, and for the slopes no
// higher than where their complements are.  (A comparison keeps a NaN.)
constexpr float kFarOut = 128.f;
__device__ __forceinline__ float not_below(float z) { return z < -kFarOut ? -kFarOut : z; }
__device__ __forceinline__ float inside(float z) { return z > kFarOut ? kFarOut : not_below(z); }

// Eight at a time: one branch on the activation for all of them.
template <class F>
__device__ __forceinline__ f32x8 each8(f32x8 z, F f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = f(z[e]);
  return z;
}
template <bool FAST>
__device__ __forceinline__ f32x8 act8(int act, f32x8 z, float slope) {
  switch (act) {
    case LIPZ_ACT_RELU: return each8(z, [](float v) { return v < 0.f ? 0.f : v; });
    case LIPZ_ACT_LRELU: return each8(z, [=](float v) { return v < 0.f ? slope * v : v; });
    case LIPZ_ACT_TANH: return each8(z, [](float v) { return tanh_of<FAST>(v); });
    case LIPZ_ACT_GELU:
      return each8(z, [](float v) {
        v = not_below(v);
        return v * normal_cdf<FAST>(v, FAST ? exp_of<true>(-0.5f * v * v) : 0.f);
      });
    case LIPZ_ACT_SILU:
      return each8(z, [](float v) {
        v = not_below(v);
        return v * recip<FAST>(1.f + exp_of<FAST>(-v));
      });
    default: return z;
  }
}
template <bool FAST>
__device__ __forceinline__ f32x8 slope8(int act, f32x8 z, float slope) {
  switch (act) {
    case LIPZ_ACT_RELU: return each8(z, [](float v) { return v > 0.f ? 1.f : (v <= 0.f ? 0.f : v); });
    case LIPZ_ACT_LRELU: return each8(z, [=](float v) { return v > 0.f ? 1.f : (v <= 0.f ? slope : v); });
    case LIPZ_ACT_TANH:
      return each8(z, [](float v) {  // 1 - tanh^2
        const float e = exp_of<FAST>(-2.f * __builtin_fabsf(v)), q = recip<FAST>(1.f + e);
        return 4.f * e * q * q;
      });
    case LIPZ_ACT_GELU:
      return each8(z, [](float v) {
        v = inside(v);
        const float e = exp_of<FAST>(-0.5f * v * v);
        return fmaf(v * kInvSqrt2Pi, e, normal_cdf<FAST>(v, e));
      });
    case LIPZ_ACT_SILU:
      return each8(z, [](float v) {
        v = inside(v);
        const float s = recip<FAST>(1.f + exp_of<FAST>(-v));
        return s * fmaf(v, 1.f - s, 1.f);
      });
    default: return each8(z, [](float) { return 1.f; });
  }
}

// ---- the host's checks ----

constexpr int64_t kMaxWide = 1 << 20;  // columns of a matrix
constexpr int kMaxCells = 65535;       // a grid's second dimension
constexpr int kMaxRows = 1 << 21;      // rows of a product

inline int elem_size(int dtype) { return dtype == LIPZ_F32 ? 4 : dtype == LIPZ_FP8 ? 1 : 2; }
inline bool valid_float(int dtype) { return dtype == LIPZ_F32 || dtype == LIPZ_BF16 || dtype == LIPZ_F16; }

// Strides and alignment of a [cells][rows][cols] matrix.  `out`: written, so
// its cells must lie apart.
inline lipz_status check_mat(const lipz_mat& m, int cells, int64_t rows, int64_t cols, int dtype, bool out) {
  if (m.ld < cols || m.cell < 0) return LIPZ_E_INVAL;
  if (m.ld > LIPZ_MAX_LD) return LIPZ_E_UNSUPPORTED;
  if ((uintptr_t)m.p % (size_t)elem_size(dtype)) return LIPZ_E_INVAL;
  if (m.cell > (INT64_MAX / 16) / cells) return LIPZ_E_INVAL;
  if (out && cells > 1 && rows > 0) {
    // cells one after the other, or side by side inside the rows
    const bool apart = m.cell >= (rows - 1) * m.ld + cols;
    const bool beside = m.cell >= cols && (int64_t)(cells - 1) * m.cell + cols <= m.ld;
    if (!apart && !beside) return LIPZ_E_INVAL;
  }
  return LIPZ_OK;
}
inline lipz_status check_vec(const float* p, int64_t cell, int cells, int64_t cols, bool out) {
  if ((uintptr_t)p % 4 || cell < 0 || cell > (INT64_MAX / 16) / cells) return LIPZ_E_INVAL;
  return out && cells > 1 && cell < cols ? LIPZ_E_INVAL : LIPZ_OK;
}
// A product's workgroups (64 x 64 outputs at least, 512 splits in all at most) and the
// threads that join its splits stay far below 2^31.
inline lipz_status check_tiles(int64_t rows, int64_t cols, int64_t cells) {
  return ((rows + 63) / 64) * ((cols + 63) / 64) * cells > (1 << 24) ? LIPZ_E_UNSUPPORTED : LIPZ_OK;
}

inline lipz_status check_workspace(const void* p, size_t have, size_t need) {
  if (!need) return LIPZ_E_INVAL;
  return !p || ((uintptr_t)p & 255) || have < need ? LIPZ_E_WORKSPACE : LIPZ_OK;
}
// out[c][j] = sum over n rows of part[c][n][cols] (norm.hip)
hipError_t launch_sum_parts(const float* part, int n, int cols, int cells, float* out, int64_t out_cell, hipStream_t s);

inline lipz_status launched() { return hipGetLastError() == hipSuccess ? LIPZ_OK : LIPZ_E_HIP; }

}  // namespace lipz
