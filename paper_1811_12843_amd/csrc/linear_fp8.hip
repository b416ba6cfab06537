// lipz_linear_fp8 and lipz_quantize_weights: the product on e4m3 operands with
// a scale per row and column (kernel: block_gemm.h), and the weights that it
// reads.
//
// The quantiser turns w [fan_in][fan_out] into rows of fan_in bytes, so that the
// product reads both operands along k.  Two launches: column maxima per block
// of rows, then, per 128 x 64 tile, the column's scale from those and the tile
// through LDS, 16 lanes writing 128 bytes of a row.  Bound by memory: w is
// read twice, the second time mostly from the Infinity Cache: 8192 x 4096 bf16 37
// us.
#include "block_gemm.h"

namespace lipz {
namespace {

constexpr int kMaxRowsPer = 256;  // rows of w whose maxima one block takes

struct QuantArgs {
  const void* w;
  uint8_t* q;
  float *scale, *part;  // part: [cells][ceil(K / 256)][N]
  int64_t w_ld, w_cell, q_ld, q_cell, scale_cell;
  int K, N;
};

// 32 lanes x 8 columns, 8 rows at a time; eight of a thread's rows in flight.
template <class T>
__global__ __launch_bounds__(256) void column_max_kernel(const QuantArgs P) {
  using Raw = typename Vec8<T>::type;
  __shared__ float top[8][256 + 8];
  const int c = blockIdx.z, lane = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int n = blockIdx.x * 256 + 8 * lane, left = P.N - n, k0 = blockIdx.y * kMaxRowsPer + r;
  f32x8 m = {};
  if (left > 0) {
    for (int i0 = 0; i0 < kMaxRowsPer / 8; i0 += 8) {
      Raw v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = k0 + 8 * (i0 + i);
        v[i] = row8_raw((const T*)P.w + c * P.w_cell + min(k, P.K - 1) * P.w_ld, n, P.N);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (rows past the last one are that one again)
        const f32x8 x = widen<T>(row8_in_place<T>(v[i], n, P.N));
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = max_nan(m[e], __builtin_fabsf(x[e]));
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) top[r][8 * lane + e] = m[e];
  __syncthreads();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= P.N) return;
  float t = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) t = max_nan(t, top[q][threadIdx.x]);
  P.part[((int64_t)c * gridDim.y + blockIdx.y) * P.N + col] = t;
}

// A block turns 128 rows x 64 columns.  LDS holds them as rows of w, in chunks
// of 8 columns whose place is xored with the row's 8-row group, so that the
// reads down a column by lanes 8 rows apart lie on different banks.
constexpr int kQuantRows = 128;
template <class T>
__global__ __launch_bounds__(256) void quantize_kernel(const QuantArgs P) {
  using Raw = typename Vec8<T>::type;
  __shared__ float top[4][64], scale[64];
  __shared__ __attribute__((aligned(16))) T tile[kQuantRows][64];
  const int c = blockIdx.z, n0 = blockIdx.x * 64, k0 = blockIdx.y * kQuantRows, t = threadIdx.x;
  const int chunks = (P.K + kMaxRowsPer - 1) / kMaxRowsPer;
  const int x = t & 7;
  Raw v[kQuantRows / 32];
#pragma unroll
  for (int i = 0; i < kQuantRows / 32; ++i) {
    const int k = k0 + 32 * i + (t >> 3);
    v[i] = row8_raw((const T*)P.w + c * P.w_cell + min(k, P.K - 1) * P.w_ld, n0 + 8 * x, P.N);
  }
  {
    const int col = t & 63, g = t >> 6;
    const LIPZ_GLOBAL float* p = as_global(P.part) + (int64_t)c * chunks * P.N + n0 + col;
    float m = 0.f;
    if (n0 + col < P.N) {
#pragma unroll 8
      for (int i = g; i < chunks; i += 4) m = max_nan(m, p[(int64_t)i * P.N]);
    }
    top[g][col] = m;
  }
#pragma unroll
  for (int i = 0; i < kQuantRows / 32; ++i) {
    const int row = 32 * i + (t >> 3);
    *(Raw*)&tile[row][8 * (x ^ ((row >> 3) & 7))] = row8_in_place<T>(v[i], n0 + 8 * x, P.N);
  }
  __syncthreads();
  if (t < 64) {
    scale[t] = fp8_scale(max_nan(max_nan(top[0][t], top[1][t]), max_nan(top[2][t], top[3][t])));
    if (blockIdx.y == 0 && n0 + t < P.N) P.scale[c * P.scale_cell + n0 + t] = scale[t];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kQuantRows / 32; ++i) {
    const int k = 8 * (t & 15), n = 16 * i + (t >> 4);  // 16 lanes write a row's 128 bytes
    if (n0 + n >= P.N || k0 + k >= P.K) continue;
    f32x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (float)tile[k + e][8 * ((n >> 3) ^ (t & 7)) + (n & 7)] / scale[n];
    store8_fp8(P.q + c * P.q_cell + (n0 + n) * P.q_ld + k0 + k, P.K - k0 - k, o);
  }
}

lipz_status check_quant(const lipz_quantize_weights_args* a) {
  if (!a || a->abi_version != LIPZ_ABI_VERSION || !valid_float(a->dtype)) return LIPZ_E_INVAL;
  lipz_status st = check_sizes(a->cells, 0, a->fan_in, a->fan_out);
  if (st) return st;
  if (!a->w.p || !a->q.p || !a->scale) return LIPZ_E_INVAL;
  if ((st = check_mat(a->w, a->cells, a->fan_in, a->fan_out, a->dtype, false))) return st;
  if ((st = check_mat(a->q, a->cells, a->fan_out, a->fan_in, LIPZ_FP8, true))) return st;
  if ((st = check_vec(a->scale, a->scale_cell, a->cells, a->fan_out, true))) return st;
  return check_tiles(a->fan_in, a->fan_out, a->cells);
}

lipz_status check_linear_fp8(const lipz_linear_fp8_args* a) {
  if (!a || a->abi_version != LIPZ_ABI_VERSION || !valid_float(a->y_dtype) || !valid_block_act(a->act, a->slope))
    return LIPZ_E_INVAL;
  lipz_status st = check_sizes(a->cells, a->rows, a->fan_in, a->fan_out);
  if (st) return st;
  if (!a->w.p || !a->w_scale || (a->rows && (!a->x.p || !a->y.p || !a->x_scale))) return LIPZ_E_INVAL;
  const int C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  if ((st = check_mat(a->x, C, M, K, LIPZ_FP8, false))) return st;
  if ((st = check_mat(a->w, C, N, K, LIPZ_FP8, false))) return st;
  if (a->residual.p && (st = check_mat(a->residual, C, M, N, a->y_dtype, false))) return st;
  if ((st = check_mat(a->y, C, M, N, a->y_dtype, true))) return st;
  if ((st = check_vec(a->x_scale, a->x_scale_cell, C, M, false))) return st;
  if ((st = check_vec(a->w_scale, a->w_scale_cell, C, N, false))) return st;
  if (a->bias && (st = check_vec(a->bias, a->bias_cell, C, N, false))) return st;
  return check_tiles(M, N, C);
}

size_t quant_bytes(const lipz_quantize_weights_args* a) {
  return 256 + ((size_t)a->cells * tiles_of(a->fan_in, kMaxRowsPer) * a->fan_out * 4 + 255) / 256 * 256;
}

template <class T>
void run_quant(const QuantArgs& P, int cells, hipStream_t s) {
  column_max_kernel<T><<<dim3(tiles_of(P.N, 256), tiles_of(P.K, kMaxRowsPer), cells), 256, 0, s>>>(P);
  quantize_kernel<T><<<dim3(tiles_of(P.N, 64), tiles_of(P.K, kQuantRows), cells), 256, 0, s>>>(P);
}

struct Fp8Layout {
  bool pack_x = false, pack_w = false;
  size_t x = 0, w = 0, sums = 0, total = 256;
  Plan plan{};
};
Fp8Layout fp8_layout(const lipz_linear_fp8_args* a) {
  Fp8Layout w;
  const int C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  if (!M) return w;
  Bump b;
  w.pack_x = !loads_as_is(a->x, K, 1, true);
  w.pack_w = !loads_as_is(a->w, K, 1, true);
  if (w.pack_x) w.x = b.take(packed_bytes(M, K, 1, C));
  if (w.pack_w) w.w = b.take(packed_bytes(N, K, 1, C));
  w.plan = plan_gemm(1, M, N, K, C);
  w.sums = b.take(w.plan.part_bytes);
  w.total = b.at + 256;
  return w;
}

template <class T>
void run_linear_fp8(const lipz_linear_fp8_args* a, void* ws, hipStream_t s) {
  const Fp8Layout w = fp8_layout(a);
  char* base = (char*)ws;
  const lipz_mat x = w.pack_x ? launch_pack<uint8_t>(a->x, base + w.x, a->rows, a->fan_in, a->cells, s) : a->x;
  const lipz_mat wt = w.pack_w ? launch_pack<uint8_t>(a->w, base + w.w, a->fan_out, a->fan_in, a->cells, s) : a->w;
  GemmArgs P{};
  set_operands(P, x, wt, 1, a->rows, a->fan_out, a->fan_in, a->cells);
  P.part = (float*)(base + w.sums);
  Finish& f = P.f;
  f.y = a->y.p, f.y_ld = a->y.ld, f.y_cell = a->y.cell;
  f.r = a->residual.p, f.r_ld = a->residual.ld, f.r_cell = a->residual.cell;
  f.bias = a->bias, f.bias_cell = a->bias_cell, f.act = a->act, f.slope = a->slope;
  f.xs = a->x_scale, f.xs_cell = a->x_scale_cell, f.ws = a->w_scale, f.ws_cell = a->w_scale_cell;
  launch_gemm<Fp8, T, true, true>(P, w.plan, s);
}

}  // namespace
}  // namespace lipz

using namespace lipz;

extern "C" {

size_t lipz_quantize_weights_workspace_bytes(const lipz_quantize_weights_args* a) {
  return check_quant(a) ? 0 : quant_bytes(a);
}

lipz_status lipz_quantize_weights(const lipz_quantize_weights_args* a, void* d_workspace, size_t workspace_bytes,
                                  void* hip_stream) {
  lipz_status st = check_quant(a);
  if (st) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, quant_bytes(a)))) return st;
  QuantArgs P{};
  P.w = a->w.p, P.w_ld = a->w.ld, P.w_cell = a->w.cell;
  P.q = (uint8_t*)a->q.p, P.q_ld = a->q.ld, P.q_cell = a->q.cell;
  P.scale = a->scale, P.scale_cell = a->scale_cell, P.part = (float*)d_workspace;
  P.K = a->fan_in, P.N = a->fan_out;
  hipStream_t s = (hipStream_t)hip_stream;
  if (a->dtype == LIPZ_F32) run_quant<float>(P, a->cells, s);
  else if (a->dtype == LIPZ_BF16) run_quant<__bf16>(P, a->cells, s);
  else run_quant<_Float16>(P, a->cells, s);
  return launched();
}

size_t lipz_linear_fp8_workspace_bytes(const lipz_linear_fp8_args* a) {
  return check_linear_fp8(a) ? 0 : fp8_layout(a).total;
}

lipz_status lipz_linear_fp8(const lipz_linear_fp8_args* a, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  lipz_status st = check_linear_fp8(a);
  if (st) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, fp8_layout(a).total))) return st;
  if (!a->rows) return LIPZ_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  if (a->y_dtype == LIPZ_F32) run_linear_fp8<float>(a, d_workspace, s);
  else if (a->y_dtype == LIPZ_BF16) run_linear_fp8<__bf16>(a, d_workspace, s);
  else run_linear_fp8<_Float16>(a, d_workspace, s);
  return launched();
}

}  // extern "C"
