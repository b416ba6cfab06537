// The matrix product behind lipz_linear, lipz_linear_backward and
// lipz_linear_fp8: out = epilogue(A B) for every cell, on the matrix cores.
//
//   out(i, j) = sum_k A(i, k) B(k, j),  0 <= i < M, 0 <= j < N, 0 <= k < K
//
// An operand is KC (k contiguous: A [M][K] or B stored [N][K]) or KM (k is the
// row: A stored [K][M], B [K][N]).
//
// A workgroup owns a BM x BN tile and walks K in slices of SB bytes per row
// through NS LDS stages.  A slice is multiplied in two parts: the second part's
// fragments are read before the first one's MFMAs and the next slice's first
// ones before the second's; one barrier per slice, between the parts, after
// which every wave holds the slice in registers and its stage takes the slice
// NS on.  Tiles of 64 and 128 rows: SB = 128 (32 k of fp32, 64 of 16 bits, 128 of
// e4m3); of 256 rows: SB = 64.  MFMAs are 16 x 16 (one 16 x 16 x 32 moves less
// between registers than a 32 x 32 x 16, and the card's power is what bounds
// large products: 8192 x 4096 x 4096 bf16 along k 212 and 229 us).
//
// LDS.  KC: a row of 128 bytes is eight 16-byte chunks, chunk c at place
// c ^ (row % 8) (of 64 bytes four, at c ^ (-(row / 4) % 4)): a 16-byte read serves
// lanes 0-3, 12-15, 20-23 and 24-27 together, and so on, and their rows then lie
// on all banks.  KM: rows of the tile's columns; the chunk index is xored with bits
// of k (km_swizzle), so that the k rows that a transposing read (16 bits) or
// four b32 reads (fp32) touch lie on different banks.  Lanes permute the
// global chunk they fetch, not the LDS address: loads go straight into LDS.
//
// Loads: buffer_load ... lds, 16 bytes a lane.  What lies past an operand is
// zeros in LDS, by the resource's extent or, at the end of K, by an offset past
// it.  That takes KC rows of whole chunks, and rows that begin and end on 4
// bytes; other operands are copied into such rows first (pack_kernel).
//
// MFMAs take the B fragment first, so that a lane ends up with four columns
// of a row; the tile then passes through LDS and is finished and stored in
// rows of 8 elements per lane.
//
// Large products are bound by the matrix cores' rate at the clock that the
// card's power leaves and by the finish, whose memory traffic overlaps no other
// tile's products (the stages take 128 KiB of LDS, so a compute unit holds one
// workgroup): 8192 x 4096 x 8192 bf16 with GELU, residual and pre 534 us (1.03
// PFLOP/s, matrix cores 48 % busy), of them 455 without residual and pre and with
// SiLU; with the finish as a loop over the wave's columns 40 us more.  e4m3 8192 x
// 8192 x 4096 with the weights' quantisation 597 us (matrix cores 40 % busy, beside
// the conversion of every fragment in every wave).
// One row: the weights' bytes, 4096 x 4096 bf16 12.5 us, 7 of them the product.
#pragma once

#include "block.h"

namespace lipz {

// The operand type of e4m3 products.  Their fragments are turned into f16, which
// holds every e4m3 value, and multiplied at fp32 accuracy.  The scaled e4m3 MFMA, at
// twice the rate, aligns its products to the largest of them before it adds them,
// so that one large product takes the low bits of all others: sums of 1024 with a
// 448 x 448 of either sign in every 64 terms and remainders between 1 and 4 came out
// up to 8.7e-5 of the sum of magnitudes and 12 % of their value off (in f16 exact).
// That costs 597 us instead of 307 at 8192 x 8192 x 4096 with the weights'
// quantisation, and 12.4 instead of 11.7 at 8 x 4096 x 8192.
struct Fp8 {};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_any;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
template <class V>
__device__ __forceinline__ V lds_get(const lds_char* p) {
  return *(const __attribute__((address_space(3))) V*)p;
}

template <class E>
struct ElemSize {
  static constexpr int value = sizeof(E);
};
template <>
struct ElemSize<Fp8> {
  static constexpr int value = 1;
};

// How a product's outputs are finished.
struct Finish {
  void *y, *pre;
  const void* r;
  int64_t y_ld, y_cell, pre_ld, pre_cell, r_ld, r_cell, bias_cell, xs_cell, ws_cell;  // in elements
  const float *bias, *xs, *ws;  // xs, ws: scales of rows and columns (e4m3)
  int act;
  float slope;
};

struct GemmArgs {
  const char *A, *B;
  int64_t a_ld, a_cell, b_ld, b_cell;  // in bytes
  int M, N, K;
  int tiles_m, tiles_n, cells, splits, per_split;  // per_split: slices of a split
  float* part;                                     // splits > 1: sums [split][cell][M][part_ld]
  int part_ld;
  Finish f;
};

constexpr uint32_t kPast = 0x80000000u;

// ---- finishing: 8 columns of a row from column n on, `left` of them inside ----
// (a residual as row8_raw loads it: finish8 puts it in place)
template <class T>
__device__ __forceinline__ typename Vec8<T>::type residual8(const Finish& f, int c, int m, int n, int cols) {
  return f.r ? row8_raw((const T*)f.r + c * f.r_cell + m * f.r_ld, n, cols) : typename Vec8<T>::type{};
}
template <class T>
__device__ __forceinline__ void finish8(const Finish& f, int c, int m, int n, int left, f32x8 v, const f32x8& bias,
                                        const f32x8& ws, typename Vec8<T>::type residual) {
  constexpr bool FAST = sizeof(T) < 4;
  if (f.xs) {
    // significands first, exponents last: the scales' own product may lie below or
    // above fp32's range where theirs with the sum does not
    const float xs = as_global(f.xs)[c * f.xs_cell + m], xm = __builtin_amdgcn_frexp_mantf(xs);
    const int xe = __builtin_amdgcn_frexp_expf(xs);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = __builtin_amdgcn_ldexpf(v[e] * (xm * __builtin_amdgcn_frexp_mantf(ws[e])),
                                     xe + __builtin_amdgcn_frexp_expf(ws[e]));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += bias[e];
  if (f.pre) store8((T*)f.pre + c * f.pre_cell + m * f.pre_ld + n, left, v);
  v = act8<FAST>(f.act, v, f.slope);
  if (f.r) {
    const f32x8 r = widen<T>(row8_in_place<T>(residual, n, n + left));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += r[e];
  }
  store8((T*)f.y + c * f.y_cell + m * f.y_ld + n, left, v);
}
__device__ __forceinline__ f32x8 column8(const float* p, int64_t cell, int c, int n, int cols) {
  return p && n < cols ? row8(p + c * cell, n, cols) : f32x8{};
}

// ---- operands ----

// The place of chunk x (16 bytes) of k row k in a KM tile of R columns is
// x ^ km_swizzle(k).  16 bits: a transposing read of a group of 16 lanes takes 32
// bytes of each of four k rows; two groups, 8 k rows apart, are served at a time.
// fp32: a read takes 64 bytes of k rows 4 g + u.
template <int ES, int R>
__device__ __forceinline__ int km_swizzle(int k) {
  if (ES == 4) return 4 * ((k >> 2) & 3);
  if (R * ES >= 256) return 2 * ((k & 3) | ((k >> 1) & 4));
  return 2 * (((k >> 1) & 1) | ((k >> 2) & 2));
}
template <int SB>
__device__ __forceinline__ int kc_swizzle(int row) {
  return SB == 128 ? row & 7 : -(row >> 2) & 3;
}

template <int ES, bool KC, int R, class Tile>
struct Operand {
  static constexpr int SB = Tile::SB, NT = Tile::NT;
  static constexpr int EPC = 16 / ES, BKE = SB / ES;
  static constexpr int NI = R * SB / 16 / NT;             // chunks of a slice per thread
  static constexpr int CPR = KC ? SB / 16 : R * ES / 16;  // chunks of an LDS row
  const char* base;  // the next slice of the tile
  int64_t step;      // bytes per slice
  int extent;        // KC: bytes from base to the end of the tile's last row; KM: bytes of the operand's columns from the tile's on
  int ld;            // KM: row pitch
  int kleft;         // k left from the next slice on
  uint32_t off[NI];  // the thread's chunks in a slice, from its base
  int k;             // KC: first k of the thread's chunks in their slice (the same in all of them)

  __device__ __forceinline__ void init(const char* p, int64_t ld_bytes, int rc0, int rc_all, int K, int k0) {
    ld = (int)ld_bytes;
    kleft = K - k0;
    if (KC) {
      base = p + (int64_t)rc0 * ld_bytes + (int64_t)k0 * ES;
      step = SB;
      extent = (min(rc_all - rc0, R) - 1) * ld + (kleft * ES + 15) / 16 * 16;  // (packed rows end in zeros)
    } else {
      base = p + (int64_t)k0 * ld_bytes + (int64_t)rc0 * ES;
      step = BKE * ld_bytes;
      extent = ((rc_all - rc0) * ES + 3) / 4 * 4;
    }
    static_assert(!KC || NT / CPR % 16 == 0, "a thread's rows have the same swizzle");
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int q = i * NT + (int)threadIdx.x, row = q / CPR, at = q % CPR;
      const int x = at ^ (KC ? kc_swizzle<SB>(row) : km_swizzle<ES, R>(row));
      off[i] = (uint32_t)row * (uint32_t)ld + x * 16;
      if (KC) k = x * EPC;
    }
  }
  // The next slice into LDS; one past the end of K is zeros.
  __device__ __forceinline__ void load(lds_char* st) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (no branches here: with one, the compiler no longer sees which stage a
    // load in flight goes to, and waits for it before it reads the other)
    const int e = KC ? max(extent, 0) : max((min(kleft, BKE) - 1) * ld + extent, 0);
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, e, 0x00020000);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t o = KC && k >= kleft ? kPast : off[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_any*)(st + (i * NT + wave * 64) * 16), 16, (int)o, 0, 0, 0);
    }
    base += step;
    kleft -= BKE;
    if (KC) extent -= SB;
  }
};

// Fragments of 16 rows (columns) from r0 on, as MFMAs take them: lane l holds
// row l % 16 and, of the slice's half kk, 16 bytes of k (16 bits: k = 32 kk +
// 8 (l / 16) .. + 7; fp32: 16 kk + 4 (l / 16) .. + 3; e4m3: 64 kk + 16 (l / 16) .. +
// 15; A and B need only agree).  N of them, 16 rows apart.
template <int ES, bool KC, int R, int SB, int N>
struct Fragments {
  static __device__ __forceinline__ void read(const lds_char* st, int r0, int kk, int lane, u32x4* out) {
    const int li = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + 16 * i + li;
      if (KC) {
        out[i] = lds_get<u32x4>(st + r * SB + (((4 * kk + g) ^ kc_swizzle<SB>(li)) << 4));
      } else {  // fp32
        const int k = 16 * kk + 4 * g;
        const lds_char* p = st + k * (R * 4) + (((r >> 2) ^ km_swizzle<4, R>(k)) << 4) + 4 * (r & 3);
#pragma unroll
        for (int u = 0; u < 4; ++u) out[i][u] = lds_get<uint32_t>(p + u * (R * 4));
      }
    }
  }
};

// 16 bits, KM, by transposing reads: in each, lane i of a group of 16 gives the
// address of four columns of k row i / 4 and receives column i of the four
// rows; a second one takes the k rows 4 on.  The two index the stage each by
// itself: the compiler follows a pointer only some steps to see which stage it
// reads, and waits for every load in flight where it no longer sees it.
__device__ __forceinline__ u32x4 read_transposed(const lds_char* st, int at, int at4) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  typedef short v8s __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) v4s lds_v4s;
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(st + at));
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(st + at4));
  return __builtin_bit_cast(u32x4, (v8s{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}));
}
__device__ __forceinline__ int hidden(int v) {
  asm("" : "+v"(v));
  return v;
}
template <int R, int SB, int N>
struct Fragments<2, false, R, SB, N> {
  static __device__ __forceinline__ void read(const lds_char* st, int r0, int kk, int lane, u32x4* out) {
    const int li = lane & 15, k = 8 * (lane >> 4) + (li >> 2);
    const int p = k * (R * 2) + 8 * (li & 1), p4 = hidden(p + 4 * R * 2);
    const int x = (r0 >> 3) + ((li >> 1) & 1), w = km_swizzle<2, R>(k);
#pragma unroll
    for (int i = 0; i < N; ++i)
      out[i] = read_transposed(st, p + (((x + 2 * i) ^ w) << 4) + kk * 32 * R * 2,
                               p4 + (((x + 2 * i) ^ w) << 4) + kk * 32 * R * 2);
  }
};

template <class E>
struct Mma;
template <>
struct Mma<__bf16> {
  static __device__ __forceinline__ f32x4 run(u32x4 b, u32x4 a, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
  }
};
template <>
struct Mma<_Float16> {
  static __device__ __forceinline__ f32x4 run(u32x4 b, u32x4 a, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
  }
};
template <>
struct Mma<float> {
  static __device__ __forceinline__ f32x4 run(u32x4 b, u32x4 a, f32x4 c) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b[u]), __uint_as_float(a[u]), c, 0, 0, 0);
    return c;
  }
};

// ---- tiles ----

template <int BM_, int BN_, int WM_, int WN_, int NS_, int SB_>
struct TileShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;  // WM x WN waves
  static constexpr int NS = NS_, SB = SB_;                      // LDS stages, bytes of a slice's row
  static constexpr int NT = 64 * WM * WN, TM = BM / WM, TN = BN / WN;
  static constexpr int MI = TM / 16, NI = TN / 16;              // MFMAs of 16 x 16
  static constexpr int A_BYTES = BM * SB, B_BYTES = BN * SB;
  static constexpr int LOADS = (A_BYTES + B_BYTES) / 16 / NT;  // of a slice, per wave
  static_assert(NS >= 2 && NS <= 4 && 2 * NS >= WM * WN && TM % 32 == 0 && TN % 32 == 0 && BM * SB >= 4096);
};
// (three stages: three workgroups to a compute unit; with four, two of them, one row of
// 4096 x 4096 bf16 13.2 us instead of 12.3, gradients at 1999 x 1201 x 777 f16 44.5
// instead of 43.4)
typedef TileShape<64, 64, 2, 2, 3, 128> TileS;
typedef TileShape<128, 128, 2, 2, 4, 128> TileM;
typedef TileShape<256, 256, 2, 4, 4, 64> TileL;

// Waits until all but this wave's last n vector loads have landed and its LDS
// accesses are done, then for the other waves.  No more than that: the
// compiler's barrier would wait for every load.
template <int n>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4 << 14) | 0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A wave's products of a slice, in two parts.  Where MFMAs take the slice's k
// in one step, a part is half of the wave's rows.
template <class E, bool AKC, bool BKC, class Tile, bool ONE_STEP>
struct Parts {
  static constexpr int ES = ElemSize<E>::value, H = Tile::MI / 2;
  u32x4 a[2][H], b[2][Tile::NI];  // B's serve both parts: b[1] are the ones of the part that is left
  __device__ __forceinline__ void turn() {
#pragma unroll
    for (int j = 0; j < Tile::NI; ++j) b[1][j] = b[0][j];
  }
  template <int P>
  __device__ __forceinline__ void read(const lds_char* sa, const lds_char* sb, int wm, int wn, int lane) {
    if (P == 0) Fragments<ES, BKC, Tile::BN, Tile::SB, Tile::NI>::read(sb, wn, 0, lane, b[0]);
    Fragments<ES, AKC, Tile::BM, Tile::SB, H>::read(sa, wm + 16 * H * P, 0, lane, a[P]);
  }
  template <int P>
  __device__ __forceinline__ void mma(f32x4 (&acc)[Tile::MI][Tile::NI]) {
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < Tile::NI; ++j) acc[H * P + i][j] = Mma<E>::run(b[P][j], a[P][i], acc[H * P + i][j]);
  }
};
// Otherwise (16 bits and fp32) half of its k.
template <class E, bool AKC, bool BKC, class Tile>
struct Parts<E, AKC, BKC, Tile, false> {
  static constexpr int ES = ElemSize<E>::value;
  struct Frag {
    u32x4 a[Tile::MI], b[Tile::NI];
  };
  Frag f[2];
  __device__ __forceinline__ void turn() {}
  template <int P>
  __device__ __forceinline__ void read(const lds_char* sa, const lds_char* sb, int wm, int wn, int lane) {
    Fragments<ES, BKC, Tile::BN, Tile::SB, Tile::NI>::read(sb, wn, P, lane, f[P].b);
    Fragments<ES, AKC, Tile::BM, Tile::SB, Tile::MI>::read(sa, wm, P, lane, f[P].a);
  }
  template <int P>
  __device__ __forceinline__ void mma(f32x4 (&acc)[Tile::MI][Tile::NI]) {
#pragma unroll
    for (int i = 0; i < Tile::MI; ++i)
#pragma unroll
      for (int j = 0; j < Tile::NI; ++j) acc[i][j] = Mma<E>::run(f[P].b[j], f[P].a[i], acc[i][j]);
  }
};

// e4m3: a part is half of the wave's rows.
template <bool AKC, bool BKC, class Tile>
struct Parts<Fp8, AKC, BKC, Tile, false> {
  static constexpr int H = Tile::MI / 2;
  u32x4 fb[2][2][Tile::NI], fa[2][2][H];  // B's serve both parts: fb[1] are the ones of the part that is left
  __device__ __forceinline__ void turn() {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int j = 0; j < Tile::NI; ++j) fb[1][kk][j] = fb[0][kk][j];
  }
  template <int P>
  __device__ __forceinline__ void read(const lds_char* sa, const lds_char* sb, int wm, int wn, int lane) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      if (P == 0) Fragments<1, true, Tile::BN, Tile::SB, Tile::NI>::read(sb, wn, kk, lane, fb[0][kk]);
      Fragments<1, true, Tile::BM, Tile::SB, H>::read(sa, wm + 16 * H * P, kk, lane, fa[P][kk]);
    }
  }
  template <int P>
  __device__ __forceinline__ void mma(f32x4 (&acc)[Tile::MI][Tile::NI]) {
    const auto& a = fa[P];
    const auto& b = fb[P];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f16x8 w[Tile::NI];
#pragma unroll
      for (int j = 0; j < Tile::NI; ++j) w[j] = eight(b[q / 2][j], q);
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const f16x8 x = eight(a[q / 2][i], q);
#pragma unroll
        for (int j = 0; j < Tile::NI; ++j)
          acc[H * P + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[j], x, acc[H * P + i][j], 0, 0, 0);
      }
    }
  }
  // bytes 8 (q % 2) .. + 7 of a fragment
  static __device__ __forceinline__ f16x8 eight(u32x4 v, int q) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    f16x8 r;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const uint32_t w = v[q % 2 * 2 + d];
      const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
      const f16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
      r[4 * d] = lo[0], r[4 * d + 1] = lo[1], r[4 * d + 2] = hi[0], r[4 * d + 3] = hi[1];
    }
    return r;
  }
};

// The tile of a workgroup.  Workgroup b runs on XCD b % 8: each XCD takes a
// contiguous share of the tiles, and tiles follow each other down `GM` rows
// and then along, so that those in flight on an XCD share rows and columns in
// its L2.
__device__ __forceinline__ void tile_of(const GemmArgs& P, int GM, int& c, int& split, int& tm, int& tn) {
  const int total = gridDim.x, q = total >> 3, r = total & 7, x = blockIdx.x & 7;
  int t = x * q + min(x, r) + (blockIdx.x >> 3);
  const int per = P.tiles_m * P.tiles_n;
  const int cs = t / per;
  t -= cs * per;
  c = cs / P.splits;
  split = cs - c * P.splits;
  const int band = GM * P.tiles_n, first = t / band * GM, rows = min(P.tiles_m - first, GM);
  t %= band;
  tm = first + t % rows;
  tn = t / rows;
}

template <class E, class T, bool AKC, bool BKC, class Tile>
__global__ __launch_bounds__(Tile::NT) void block_gemm_kernel(const GemmArgs P) {
  constexpr int ES = ElemSize<E>::value, BKE = Tile::SB / ES;
  // separate arrays: a load into one stage is then seen not to touch the
  // others, and reads of those do not wait for it
  constexpr int NS = Tile::NS;
  struct Stage {
    lds_char *a, *b;
  };
#define LIPZ_STAGE(i)                                                                               \
  __shared__ __attribute__((aligned(1024))) char ldsa##i[NS > i ? Tile::A_BYTES : 16];              \
  __shared__ __attribute__((aligned(1024))) char ldsb##i[NS > i ? Tile::B_BYTES : 16];              \
  const Stage stage##i = {(lds_char*)ldsa##i, (lds_char*)ldsb##i};
  LIPZ_STAGE(0)
  LIPZ_STAGE(1)
  LIPZ_STAGE(2)
  LIPZ_STAGE(3)
#undef LIPZ_STAGE
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / Tile::WN * Tile::TM, wn = wave % Tile::WN * Tile::TN;
  int c, split, tm, tn;
  tile_of(P, 4, c, split, tm, tn);
  const int m0 = tm * Tile::BM + wm, n0 = tn * Tile::BN + wn;  // the wave's block
  const int k0 = split * P.per_split * BKE, kend = min(P.K, k0 + P.per_split * BKE);
  Operand<ES, AKC, Tile::BM, Tile> A;
  Operand<ES, BKC, Tile::BN, Tile> B;
  A.init(P.A + c * P.a_cell, P.a_ld, tm * Tile::BM, P.M, kend, k0);
  B.init(P.B + c * P.b_cell, P.b_ld, tn * Tile::BN, P.N, kend, k0);
  auto load = [&](const Stage& st) {
    A.load(st.a);
    B.load(st.b);
  };
  load(stage0);
  load(stage1);
  if constexpr (NS > 2) load(stage2);
  if constexpr (NS > 3) load(stage3);
  f32x4 acc[Tile::MI][Tile::NI] = {};
  Parts<E, AKC, BKC, Tile, ES == 2 && Tile::SB == 64> F;
  // Keeps the order that is written, where registers allow it (both operands
  // across k take more addresses): 6 cold 8192 x 4096 x 4096 products along k
  // 1383 us, 1475 in the compiler's order.
  auto pin = [] {
    if constexpr (AKC) __builtin_amdgcn_sched_barrier(0);
  };
  // One slice, in `cur`, its first part's fragments in registers.
  auto step = [&](const Stage& cur, const Stage& next) {
    F.template read<1>(cur.a, cur.b, wm, wn, lane);
    pin();
    F.template mma<0>(acc);
    pin();
    wait_and_meet<(NS - 2) * Tile::LOADS>();  // the next slice is in LDS, and every wave has read this one
    load(cur);
    F.turn();
    F.template read<0>(next.a, next.b, wm, wn, lane);
    pin();
    F.template mma<1>(acc);
    pin();
  };
  const Stage& last = NS == 2 ? stage1 : NS == 3 ? stage2 : stage3;

  int slices = (kend - k0 + BKE - 1) / BKE;
  wait_and_meet<(NS - 1) * Tile::LOADS>();
  F.template read<0>(stage0.a, stage0.b, wm, wn, lane);
  for (; slices >= NS; slices -= NS) {
    step(stage0, stage1);
    if constexpr (NS > 2) step(stage1, stage2);
    if constexpr (NS > 3) step(stage2, stage3);
    step(last, stage0);
  }
  if (slices > 0) step(stage0, stage1);
  if constexpr (NS > 2)
    if (slices > 1) step(stage1, stage2);
  if constexpr (NS > 3)
    if (slices > 2) step(stage2, stage3);
  wait_and_meet<0>();

  // The wave's block, 32 x 32 of it at a time: a lane's columns pass through
  // LDS, chunk x of a row (16 bytes) at place x ^ (row % 8), and come back as
  // 8 columns of one row, 16 rows at a time.
  const bool sums = P.splits > 1;
  float* part = P.part + ((int64_t)split * P.cells + c) * P.M * P.part_ld;
  const int at_stage = wave % NS;
  const Stage& own = at_stage == 0 ? stage0 : at_stage == 1 ? stage1 : at_stage == 2 ? stage2 : stage3;
  lds_char* mine = wave < NS ? own.a : own.b;
#pragma unroll
  for (int bj = 0; bj < Tile::TN / 32; ++bj) {
    const int n = n0 + 32 * bj + 8 * (lane & 3), left = P.N - n;
    const f32x8 bias = sums ? f32x8{} : column8(P.f.bias, P.f.bias_cell, c, n, P.N);
    const f32x8 ws = sums ? f32x8{} : column8(P.f.ws, P.f.ws_cell, c, n, P.N);
    // all of the columns' residuals now: a load is waited for together with the stores before it
    typename Vec8<T>::type r[Tile::TM / 32][2] = {};
    if (P.f.r && !sums) {
#pragma unroll
      for (int bi = 0; bi < Tile::TM / 32; ++bi)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          r[bi][p] = residual8<T>(P.f, c, min(m0 + 32 * bi + 16 * p + (lane >> 2), P.M - 1), n, P.N);
        }
    }
#pragma unroll
    for (int bi = 0; bi < Tile::TM / 32; ++bi) {
      const int row = lane >> 2, m = m0 + 32 * bi + row;
      // C of a 16 x 16 MFMA: lane l holds row l % 16, columns 4 (l / 16) .. + 3
      auto put = [&](int at, int x, f32x4 v) { *(lds_f32x4*)(mine + at * 128 + ((x ^ (at & 7)) << 4)) = v; };
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) put(16 * i + (lane & 15), 4 * j + (lane >> 4), acc[2 * bi + i][2 * bj + j]);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int at = row + 16 * p, x = 2 * (lane & 3);
        const f32x4 lo = lds_get<f32x4>(mine + at * 128 + ((x ^ (at & 7)) << 4));
        const f32x4 hi = lds_get<f32x4>(mine + at * 128 + (((x + 1) ^ (at & 7)) << 4));
        const f32x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (m + 16 * p < P.M && left > 0) {
          if (sums) store8(part + (int64_t)(m + 16 * p) * P.part_ld + n, 8, v);
          else finish8<T>(P.f, c, m + 16 * p, n, left, v, bias, ws, r[bi][p]);
        }
      }
      // the reads are issued before the next block's writes, and LDS runs a
      // wave's accesses in order
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// The splits' sums, in order, and the finish.  A thread takes 8 columns of a row.
template <class T>
__global__ __launch_bounds__(256) void join_splits_kernel(const GemmArgs P) {
  const int per_row = P.part_ld / 8;
  const int64_t rows = (int64_t)P.cells * P.M;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= rows * per_row) return;
  const int64_t row = at / per_row;
  const int n = 8 * (int)(at - row * per_row), c = (int)(row / P.M), m = (int)(row - (int64_t)c * P.M), left = P.N - n;
  const float* p = P.part + row * P.part_ld + n;
  f32x8 v = {};
  // eight splits' sums in flight; past the last split the last one again, not added
  for (int s0 = 0; s0 < P.splits; s0 += 8) {
    f32x8 w[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) w[u] = load8(p + min(s0 + u, P.splits - 1) * rows * P.part_ld, 8);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (s0 + u < P.splits) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[u][e];
      }
  }
  finish8<T>(P.f, c, m, n, left, v, column8(P.f.bias, P.f.bias_cell, c, n, P.N),
             column8(P.f.ws, P.f.ws_cell, c, n, P.N), residual8<T>(P.f, c, m, n, P.N));
}

// ---- the host's checks, operands and workspaces ----

inline bool valid_block_act(int a, float slope) {
  return a >= LIPZ_ACT_LINEAR && a <= LIPZ_ACT_SILU && (a != LIPZ_ACT_LRELU || (slope > 0.f && slope < __builtin_inff()));
}

inline lipz_status check_sizes(int cells, int rows, int fan_in, int fan_out) {
  if (cells < 1 || rows < 0 || fan_in < 1 || fan_out < 1) return LIPZ_E_INVAL;
  if (cells > kMaxCells || rows > kMaxRows || fan_in > kMaxWide || fan_out > kMaxWide) return LIPZ_E_UNSUPPORTED;
  return LIPZ_OK;
}

inline void set_operands(GemmArgs& P, const lipz_mat& A, const lipz_mat& B, int es, int M, int N, int K, int cells) {
  P.A = (const char*)A.p, P.a_ld = A.ld * es, P.a_cell = A.cell * es;
  P.B = (const char*)B.p, P.b_ld = B.ld * es, P.b_cell = B.cell * es;
  P.M = M, P.N = N, P.K = K, P.cells = cells;
}

// A workspace's parts, each from a multiple of 256 bytes on.
struct Bump {
  size_t at = 0;
  size_t take(size_t n) {
    const size_t p = at;
    at += (n + 255) / 256 * 256;
    return p;
  }
};

// Whether an operand [rows][cols] can go straight into LDS; kc: k along its rows.
inline bool loads_as_is(const lipz_mat& m, int64_t cols, int es, bool kc) {
  return ((uintptr_t)m.p & 3) == 0 && (m.ld * es) % 4 == 0 && (m.cell * es) % 4 == 0 && (cols * es) % (kc ? 16 : 4) == 0;
}
inline int64_t packed_ld(int64_t cols, int es) { return (cols * es + 63) / 64 * 64 / es; }
inline size_t packed_bytes(int64_t rows, int64_t cols, int es, int cells) {
  return (size_t)cells * rows * packed_ld(cols, es) * es;
}

// Copies [cells][rows][cols] into rows of whole 64-byte blocks (dst, zeros past
// cols).  W: an unsigned integer of the elements' size.
template <class W>
__global__ __launch_bounds__(256) void pack_kernel(const W* src, int64_t ld, int64_t cell, W* dst, int64_t dst_ld, int rows,
                                                   int cols) {
  constexpr int EPC = 16 / (int)sizeof(W);
  struct __attribute__((packed, aligned(sizeof(W)))) Chunk {
    u32x4 v;
  };
  const int per = (int)dst_ld / EPC;
  const int64_t n = (int64_t)rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int col = (int)(i - row * per) * EPC, left = cols - col;
    const LIPZ_GLOBAL W* p = as_global(src) + blockIdx.y * cell + row * ld + col;
    u32x4 w = {};
    if (left >= EPC) {
      w = reinterpret_cast<const LIPZ_GLOBAL Chunk*>(p)->v;
    } else {
#pragma unroll
      for (int e = 0; e < EPC - 1; ++e)
        if (e < left) w[e * (int)sizeof(W) / 4] |= (uint32_t)p[e] << (8 * (e * (int)sizeof(W) % 4));
    }
    *reinterpret_cast<LIPZ_GLOBAL u32x4*>(as_global(dst) + ((int64_t)blockIdx.y * rows + row) * dst_ld + col) = w;
  }
}
template <class W>
inline lipz_mat launch_pack(const lipz_mat& m, void* dst, int rows, int cols, int cells, hipStream_t s) {
  const int64_t ld = packed_ld(cols, sizeof(W)), chunks = (int64_t)rows * ld * sizeof(W) / 16;
  const int64_t blocks = (chunks + 255) / 256, most = 4096 / cells + 1;
  pack_kernel<W><<<dim3((unsigned)(blocks < most ? blocks : most), cells), 256, 0, s>>>((const W*)m.p, m.ld, m.cell, (W*)dst, ld,
                                                                                    rows, cols);
  return lipz_mat{dst, ld, rows * ld};
}

// ---- the host's choices ----

template <class E>
constexpr bool kLarge = !std::is_same_v<E, float> && !std::is_same_v<E, Fp8>;

enum { TILE_S = 0, TILE_M = 1, TILE_L = 2 };
struct Plan {
  int tile, splits, per_split;
  size_t part_bytes;
};

inline int tiles_of(int n, int b) { return (n + b - 1) / b; }
inline int tile_size(int tile) { return tile == TILE_L ? 256 : tile == TILE_M ? 128 : 64; }

// What a wave of 256 tiles takes, one to a compute unit, in microseconds: fixed (the
// pipeline's fill, the finish) and per 2048 bytes of a row of k.  Fits, to a tenth, of
// 256 .. 8192 x 4096 outputs at k = 64 .. 4096, each tile alone on all of them; e.g.
// 8192 x 4096, k = 4096 (16 bits 392, 334, 225 us; fp32 2054, 2201; e4m3 293, 304) and
// k = 64 (48, 58, 37; 90, 114; 56, 73).
struct TileTime {
  double fixed, per_2k;
};
inline const TileTime* tile_times(int es) {
  static constexpr TileTime k32[] = {{1.5, 7.85}, {8, 33.3}}, k16[] = {{0.9, 2.75}, {6, 8.8}, {15, 24}},
                            k8[] = {{1.1, 4.05}, {8, 14.7}};
  return es == 4 ? k32 : es == 2 ? k16 : k8;
}

// The tile whose whole waves take the least time by the table; of times within a
// tenth the larger tile's, which reads its operands less often.  16 bits, 64 / 128 /
// 256: 48 cells of 300 x 260, k = 1032 27 / 33 / 38 us (taken: 64), 32 cells of 130 x
// 2048, k = 512 31 / 45 / 28 (256), 1000 x 4096, k = 4096 59 / 43 / 92 (128).  fp32: 32
// cells of 10 x 2048, k = 512 51 / 79 (64), 16 of 100 x 2048, k = 1024 92 / 80 (128).
// e4m3: 8192 x 4096, k = 8192 584 / 530 (128), 2500 x 2000, k = 2048 30 / 47 (64).  Not
// seen by it: few rows bound by their weights' bytes, 16 cells of 64 x 4096, k = 1024
// bf16 35 / 38 / 31 (64).
inline int choose_tile(int es, int M, int N, int K, int cells) {
  const TileTime* times = tile_times(es);
  int tile = TILE_S;
  double best = 0;
  for (int t = TILE_S; t <= (es == 2 ? TILE_L : TILE_M); ++t) {
    const int64_t tiles = (int64_t)tiles_of(M, tile_size(t)) * tiles_of(N, tile_size(t)) * cells;
    const double us = (double)((tiles + 255) / 256) * (times[t].fixed + times[t].per_2k * ((double)K * es / 2048));
    // (a grid has less than 2^32 threads)
    if (t == TILE_S || us < 1.1 * best || (tile == TILE_S && tiles > 1 << 21)) tile = t;
    if (t == TILE_S || us < best) best = us;
  }
  return tile;
}

inline Plan plan_gemm(int es, int M, int N, int K, int cells) {
  Plan p{choose_tile(es, M, N, K, cells), 1, 0, 0};
  const int b = tile_size(p.tile);
  const int64_t tiles = (int64_t)tiles_of(M, b) * tiles_of(N, b) * cells;
  const int slices = tiles_of(K * es, p.tile == TILE_L ? 64 : 128);
  int splits = 1;
  if (p.tile == TILE_S && tiles < 256) {
    splits = (int)(512 / tiles);
    if (splits > slices / 4) splits = slices / 4;
    if (splits < 1) splits = 1;
  }
  p.per_split = tiles_of(slices, splits);
  p.splits = tiles_of(slices, p.per_split);
  if (p.splits > 1) p.part_bytes = (size_t)p.splits * cells * M * (size_t)((N + 7) / 8 * 8) * 4;
  return p;
}

template <class E, class T, bool AKC, bool BKC>
inline void launch_gemm(GemmArgs& P, const Plan& plan, hipStream_t s) {
  const int b = tile_size(plan.tile);
  P.tiles_m = tiles_of(P.M, b);
  P.tiles_n = tiles_of(P.N, b);
  P.splits = plan.splits;
  P.per_split = plan.per_split;
  P.part_ld = (P.N + 7) / 8 * 8;
  const dim3 grid((unsigned)(P.tiles_m * P.tiles_n * P.cells * P.splits));
#define LIPZ_TILE(ID, TILE) \
  if (plan.tile == ID) block_gemm_kernel<E, T, AKC, BKC, TILE><<<grid, TILE::NT, 0, s>>>(P);
  LIPZ_TILE(TILE_S, TileS)
  LIPZ_TILE(TILE_M, TileM)
  if constexpr (kLarge<E>) {
    LIPZ_TILE(TILE_L, TileL)
  }
#undef LIPZ_TILE
  if (P.splits > 1) {
    const int64_t threads = (int64_t)P.cells * P.M * (P.part_ld / 8);
    join_splits_kernel<T><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, s>>>(P);
  }
}

}  // namespace lipz
