// lipz_linear and lipz_linear_backward: matrix products with bias, activation
// and residual in the epilogue, and their gradients (kernel: block_gemm.h).
//
// Backward: one pass forms dz = dy act'(pre), rounds it to the operands' type
// for the two products (matrix cores take no wider operand beside a 16-bit one,
// and fp32 products run at a seventh of the rate; large bf16 gradients are then
// 2.3e-3 off in the 2-norm instead of their own rounding's 1.7e-3), which take it
// from L2 or the Infinity Cache, and sums its columns, unrounded, per 32 rows; a second adds those for db.  dx =
// dz w^T reads both operands along k; dw = x^T dz both across it.
// At 8192 x 4096 x 4096 bf16, 488 to 500 us together: dz 38 to 44 us (201 MB, 4.6
// TB/s and more), the products 249 and 215 us (1.1 and 1.3 PFLOP/s).
#include "block_gemm.h"

namespace lipz {
namespace {

// Rows of dz that a block sums.  32 rather than 64: 1999 x 777 f16 7 us instead
// of 13.  (Blocks of a cell: under 2^24, by check_tiles.)
constexpr int kRowsPer = 32;

struct SlopeArgs {
  const void *dy, *pre;
  void* dz;     // [..][dz_ld], zeros past N; NULL: only the sums
  float* part;  // [cells][ceil(M / 32)][N], NULL without db
  int64_t dy_ld, dy_cell, pre_ld, pre_cell, dz_ld, dz_cell;
  int M, N, act;
  float slope;
};

// 32 lanes x 8 columns, 8 rows at a time; four of a thread's rows in flight.
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs P) {
  using Raw = typename Vec8<T>::type;
  __shared__ float sums[8][256 + 8];
  const int c = blockIdx.y, lane = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int wide = (P.N + 255) / 256, chunk = blockIdx.x / wide, n0 = (blockIdx.x - chunk * wide) * 256;
  const int n = n0 + 8 * lane, left = P.N - n, m0 = chunk * kRowsPer + r;
  const bool slopes = P.act != LIPZ_ACT_LINEAR;
  f32x8 s = {};
  if (left > 0 || (P.dz && n < P.dz_ld)) {
#pragma unroll
    for (int i0 = 0; i0 < kRowsPer / 8; i0 += 4) {
      Raw d[4], z[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = min(m0 + 8 * (i0 + i), P.M - 1);
        d[i] = row8_raw((const T*)P.dy + c * P.dy_cell + m * P.dy_ld, n, P.N);
        z[i] = slopes ? row8_raw((const T*)P.pre + c * P.pre_cell + m * P.pre_ld, n, P.N) : Raw{};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = m0 + 8 * (i0 + i);
        f32x8 v = widen<T>(row8_in_place<T>(d[i], n, P.N));
        if (slopes) {
          const f32x8 w = slope8<(sizeof(T) < 4)>(P.act, widen<T>(row8_in_place<T>(z[i], n, P.N)), P.slope);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= w[e];
          if (left < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : 0.f;
          }
        }
        if (m < P.M) {
          if (P.dz) store8((T*)P.dz + c * P.dz_cell + m * P.dz_ld + n, 8, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e] += v[e];
        }
      }
    }
  }
  if (!P.part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[r][8 * lane + e] = s[e];
  __syncthreads();
  const int col = n0 + threadIdx.x;
  if (col >= P.N) return;
  float t = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) t += sums[q][threadIdx.x];
  P.part[((int64_t)c * (gridDim.x / wide) + chunk) * P.N + col] = t;
}

lipz_status check_linear(const lipz_linear_args* a) {
  if (!a || a->abi_version != LIPZ_ABI_VERSION || !valid_float(a->dtype) || !valid_block_act(a->act, a->slope))
    return LIPZ_E_INVAL;
  lipz_status st = check_sizes(a->cells, a->rows, a->fan_in, a->fan_out);
  if (st) return st;
  if (!a->w.p || (a->rows && (!a->x.p || !a->y.p))) return LIPZ_E_INVAL;
  const int C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  if ((st = check_mat(a->x, C, M, K, a->dtype, false))) return st;
  if ((st = check_mat(a->w, C, K, N, a->dtype, false))) return st;
  if (a->residual.p && (st = check_mat(a->residual, C, M, N, a->dtype, false))) return st;
  if (a->pre.p && (st = check_mat(a->pre, C, M, N, a->dtype, true))) return st;
  if ((st = check_mat(a->y, C, M, N, a->dtype, true))) return st;
  if (a->bias && (st = check_vec(a->bias, a->bias_cell, C, N, false))) return st;
  return check_tiles(M, N, C);
}

lipz_status check_linear_bwd(const lipz_linear_backward_args* a) {
  if (!a || a->abi_version != LIPZ_ABI_VERSION || !valid_float(a->dtype) || !valid_block_act(a->act, a->slope))
    return LIPZ_E_INVAL;
  lipz_status st = check_sizes(a->cells, a->rows, a->fan_in, a->fan_out);
  if (st) return st;
  const int C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  if (M && !a->dx.p && !a->dw.p && !a->db) return LIPZ_E_INVAL;
  if (M && (!a->dy.p || (a->act != LIPZ_ACT_LINEAR && !a->pre.p) || (a->dw.p && !a->x.p))) return LIPZ_E_INVAL;
  if (a->dx.p && !a->w.p) return LIPZ_E_INVAL;
  if ((st = check_mat(a->dy, C, M, N, a->dtype, false))) return st;
  if (a->act != LIPZ_ACT_LINEAR && (st = check_mat(a->pre, C, M, N, a->dtype, false))) return st;
  if (a->dx.p && ((st = check_mat(a->w, C, K, N, a->dtype, false)) || (st = check_mat(a->dx, C, M, K, a->dtype, true))))
    return st;
  if (a->dw.p && ((st = check_mat(a->x, C, M, K, a->dtype, false)) || (st = check_mat(a->dw, C, K, N, a->dtype, true))))
    return st;
  if (a->db && (st = check_vec(a->db, a->db_cell, C, N, true))) return st;
  if ((a->dx.p && (st = check_tiles(M, K, C))) || (a->dw.p && (st = check_tiles(K, N, C)))) return st;
  return check_tiles(M, N, C);
}

template <class T>
using Bits = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;

struct FwdLayout {
  bool pack_x = false, pack_w = false;
  size_t x = 0, w = 0, sums = 0, total = 256;
  Plan plan{};
};
FwdLayout fwd_layout(const lipz_linear_args* a) {
  FwdLayout w;
  const int es = elem_size(a->dtype), C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  if (!M) return w;
  Bump b;
  w.pack_x = !loads_as_is(a->x, K, es, true);
  w.pack_w = !loads_as_is(a->w, N, es, false);
  if (w.pack_x) w.x = b.take(packed_bytes(M, K, es, C));
  if (w.pack_w) w.w = b.take(packed_bytes(K, N, es, C));
  w.plan = plan_gemm(es, M, N, K, C);
  w.sums = b.take(w.plan.part_bytes);
  w.total = b.at + 256;
  return w;
}

template <class T>
void run_linear(const lipz_linear_args* a, void* ws, hipStream_t s) {
  constexpr int es = sizeof(T);
  const FwdLayout w = fwd_layout(a);
  char* base = (char*)ws;
  const lipz_mat x = w.pack_x ? launch_pack<Bits<T>>(a->x, base + w.x, a->rows, a->fan_in, a->cells, s) : a->x;
  const lipz_mat wt = w.pack_w ? launch_pack<Bits<T>>(a->w, base + w.w, a->fan_in, a->fan_out, a->cells, s) : a->w;
  GemmArgs P{};
  set_operands(P, x, wt, es, a->rows, a->fan_out, a->fan_in, a->cells);
  P.part = (float*)(base + w.sums);
  Finish& f = P.f;
  f.y = a->y.p, f.y_ld = a->y.ld, f.y_cell = a->y.cell;
  f.pre = a->pre.p, f.pre_ld = a->pre.ld, f.pre_cell = a->pre.cell;
  f.r = a->residual.p, f.r_ld = a->residual.ld, f.r_cell = a->residual.cell;
  f.bias = a->bias, f.bias_cell = a->bias_cell, f.act = a->act, f.slope = a->slope;
  launch_gemm<T, T, true, false>(P, w.plan, s);
}

// The backward pass's workspace: dz (also a linear layer's dy, if the products
// cannot read that as it is), packed operands, db's partial sums, the
// splits' sums.  dz's rows are whole slices, so that it serves both products.
struct BwdLayout {
  bool copy_dz = false, pack_x = false, pack_w = false;
  size_t dz = 0, x = 0, w = 0, part = 0, sums = 0, total = 256;
  int64_t dz_ld = 0;
  int chunks = 0;
  Plan dx{}, dw{};
};
BwdLayout bwd_layout(const lipz_linear_backward_args* a) {
  BwdLayout w;
  const int es = elem_size(a->dtype), C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  if (!M) return w;
  Bump b;
  w.dz_ld = packed_ld(N, es);
  w.chunks = tiles_of(M, kRowsPer);
  w.copy_dz = (a->dx.p || a->dw.p) && (a->act != LIPZ_ACT_LINEAR || !loads_as_is(a->dy, N, es, true));
  w.pack_w = a->dx.p && !loads_as_is(a->w, N, es, true);
  w.pack_x = a->dw.p && !loads_as_is(a->x, K, es, false);
  if (w.copy_dz) w.dz = b.take(packed_bytes(M, N, es, C));
  if (w.pack_x) w.x = b.take(packed_bytes(M, K, es, C));
  if (w.pack_w) w.w = b.take(packed_bytes(K, N, es, C));
  if (a->db) w.part = b.take((size_t)C * w.chunks * N * 4);
  w.dx = plan_gemm(es, M, K, N, C);
  w.dw = plan_gemm(es, K, N, M, C);
  const size_t x = a->dx.p ? w.dx.part_bytes : 0, d = a->dw.p ? w.dw.part_bytes : 0;
  w.sums = b.take(x > d ? x : d);
  w.total = b.at + 256;
  return w;
}

// rows = 0: the sums over no rows
template <class T>
__global__ __launch_bounds__(256) void clear_kernel(T* p, int64_t ld, int64_t cell, int rows, int cols) {
  const int64_t n = (int64_t)rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    p[blockIdx.y * cell + i / cols * ld + i % cols] = (T)0.f;
}

template <class T>
lipz_status run_linear_bwd(const lipz_linear_backward_args* a, void* ws, hipStream_t s) {
  constexpr int es = sizeof(T);
  const int C = a->cells, M = a->rows, K = a->fan_in, N = a->fan_out;
  char* base = (char*)ws;
  if (!M) {
    if (a->dw.p) clear_kernel<T><<<dim3(256, C), 256, 0, s>>>((T*)a->dw.p, a->dw.ld, a->dw.cell, K, N);
    if (a->db) clear_kernel<float><<<dim3(16, C), 256, 0, s>>>(a->db, N, a->db_cell, 1, N);
    return launched();
  }
  const BwdLayout w = bwd_layout(a);
  lipz_mat dz = a->dy;
  if (w.copy_dz) dz = lipz_mat{base + w.dz, w.dz_ld, M * w.dz_ld};
  if (a->db || w.copy_dz) {
    SlopeArgs S{};
    S.dy = a->dy.p, S.dy_ld = a->dy.ld, S.dy_cell = a->dy.cell;
    S.pre = a->pre.p, S.pre_ld = a->pre.ld, S.pre_cell = a->pre.cell;
    S.dz = w.copy_dz ? dz.p : nullptr, S.dz_ld = dz.ld, S.dz_cell = dz.cell;
    S.part = a->db ? (float*)(base + w.part) : nullptr;
    S.M = M, S.N = N, S.act = a->act, S.slope = a->slope;
    slope_kernel<T><<<dim3(w.chunks * tiles_of(N, 256), C), 256, 0, s>>>(S);
    if (a->db && launch_sum_parts(S.part, w.chunks, N, C, a->db, a->db_cell, s) != hipSuccess) return LIPZ_E_HIP;
  }
  if (a->dx.p) {
    const lipz_mat wt = w.pack_w ? launch_pack<Bits<T>>(a->w, base + w.w, K, N, C, s) : a->w;
    GemmArgs P{};
    set_operands(P, dz, wt, es, M, K, N, C);
    P.part = (float*)(base + w.sums);
    P.f.y = a->dx.p, P.f.y_ld = a->dx.ld, P.f.y_cell = a->dx.cell;
    launch_gemm<T, T, true, true>(P, w.dx, s);
  }
  if (a->dw.p) {
    const lipz_mat x = w.pack_x ? launch_pack<Bits<T>>(a->x, base + w.x, M, K, C, s) : a->x;
    GemmArgs P{};
    set_operands(P, x, dz, es, K, N, M, C);
    P.part = (float*)(base + w.sums);
    P.f.y = a->dw.p, P.f.y_ld = a->dw.ld, P.f.y_cell = a->dw.cell;
    launch_gemm<T, T, false, false>(P, w.dw, s);
  }
  return launched();
}

}  // namespace
}  // namespace lipz

using namespace lipz;

extern "C" {

size_t lipz_linear_workspace_bytes(const lipz_linear_args* a) {
  if (check_linear(a)) return 0;
  return fwd_layout(a).total;
}

lipz_status lipz_linear(const lipz_linear_args* a, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  lipz_status st = check_linear(a);
  if (st) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, lipz_linear_workspace_bytes(a)))) return st;
  if (!a->rows) return LIPZ_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  if (a->dtype == LIPZ_F32) run_linear<float>(a, d_workspace, s);
  else if (a->dtype == LIPZ_BF16) run_linear<__bf16>(a, d_workspace, s);
  else run_linear<_Float16>(a, d_workspace, s);
  return launched();
}

size_t lipz_linear_backward_workspace_bytes(const lipz_linear_backward_args* a) {
  return check_linear_bwd(a) ? 0 : bwd_layout(a).total;
}

lipz_status lipz_linear_backward(const lipz_linear_backward_args* a, void* d_workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  lipz_status st = check_linear_bwd(a);
  if (st) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, bwd_layout(a).total))) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  if (a->dtype == LIPZ_F32) return run_linear_bwd<float>(a, d_workspace, s);
  if (a->dtype == LIPZ_BF16) return run_linear_bwd<__bf16>(a, d_workspace, s);
  return run_linear_bwd<_Float16>(a, d_workspace, s);
}

}  // extern "C"
