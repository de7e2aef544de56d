// Host side of spark_qk_norm_rope_*: argument checks, launch shapes, dispatch.
#pragma once
#include "host_util.hpp"
#include "qk_norm_rope.hpp"

namespace {

// A tensor of the operator: any strides that keep rows 16-byte aligned and apart; the stride of an index with one value
// does not matter.  Offsets are 64 bits wide, so a cache of any length will do.
int check_rows(const spark_strides_t* s, int B, int H, int N, int d, bool is_output, TensorMap* out) {
  if (!s) return SPARK_ERR_NULL;
  const TensorMap m{B > 1 ? s->batch : 0, H > 1 ? s->head : 0, N > 1 ? s->row : d};
  if (m.batch < 0 || m.head < 0 || m.row < d) return SPARK_ERR_SHAPE;
  if (is_output && ((B > 1 && m.batch == 0) || (H > 1 && m.head == 0))) return SPARK_ERR_SHAPE;
  if ((m.batch | m.head | m.row) & 7) return SPARK_ERR_ALIGN;
  *out = m;
  return SPARK_OK;
}

// Everything but the tensors' strides.  `rows`: query and key heads' vectors.
int make_qk(QkNormRope* a, int B, int N, int H, int Hkv, int d, int rd, int table, float eps, int w_fp32, int dtype) {
  if (dtype != SPARK_F16 && dtype != SPARK_BF16) return SPARK_ERR_DTYPE;
  if (B < 1 || N < 1 || H < 1 || Hkv < 1 || d < 8 || d > 128 || (d & 7)) return SPARK_ERR_SHAPE;
  if (rd < 0 || rd > d || (rd & 7) || (rd > 0 && table < 1)) return SPARK_ERR_SHAPE;
  if (!isfinite(eps) || !(eps > 0.f)) return SPARK_ERR_SHAPE;
  // token indices, with a stride of the grid added, in 31 bits; a group of heads per row of the grid
  if ((int64_t)B * N >= (int64_t)1 << 30 || H > 32768 || Hkv > 32768) return SPARK_ERR_SHAPE;
  a->tokens = B * N; a->N = N; a->H = H; a->Hkv = Hkv; a->d = d; a->rd = rd; a->table = table;
  a->eps = eps; a->inv_d = 1.0f / (float)d; a->w_is_fp32 = w_fp32 != 0;
  return SPARK_OK;
}

// Elements of a lane's two chunks: eight where all pairs and the columns behind them come in eights.
int qk_vec(int d, int rd) { return d % 16 == 0 && rd % 16 == 0 ? 8 : 4; }
// Lanes of a row: 4 rows' widths of 64 and 128 columns.
int qk_lanes(int d, int vec) { return (d <= 64 ? 64 : 128) / (2 * vec); }

// Heads of a workgroup: as many as leave three workgroups to a CU, in the backward, whose rows are twice as many, one and a half.
// (us, at least 512 / 768 / 960 / 1500 workgroups: forward 8192 x 32 heads of 128 28.2 / 27.4 / 27.6 / 30.3, 3 x 1333 x 16 of 80 8.2 /
// 8.2 / 8.1 / 10.5; steps with 256 / 384 / 512 / 960 in the backward: 3 x 1333 x 16 of 80 22.1 / 20.6 / 22.8 / 26.3, 4096 x 40 of 128
// 48.1 / 47.5 / 49.4 / 52.9, 16384 x 40 of 64 83.6 / 82.4 / 82.4 / 87.4.)
int qk_group(const QkNormRope& a, int token_blocks, bool backward) {
  const int least = backward ? 384 : 768;
  int group = 16;
  while (group > 1 && (int64_t)token_blocks * ((a.H + group - 1) / group + (a.Hkv + group - 1) / group) < least) group /= 2;
  return group;
}

struct QkGrid {
  int x, y;
};
QkGrid qk_grid(QkNormRope* a, bool backward) {
  const int vec = qk_vec(a->d, a->rd), slots = 256 / qk_lanes(a->d, vec);
  const int token_blocks = (int)(((int64_t)a->tokens + slots - 1) / slots);
  a->group = qk_group(*a, token_blocks, backward);
  a->q_groups = (a->H + a->group - 1) / a->group;
  const int y = a->q_groups + (a->Hkv + a->group - 1) / a->group;
  if (!backward) return QkGrid{token_blocks, y};
  // a workgroup leaves one row of sums for dw: eight workgroups to a CU walk the tokens
  const int most = y < 2048 ? 2048 / y : 1;
  return QkGrid{token_blocks < most ? token_blocks : most, y};
}

template <typename T, int VEC, int LPR>
int launch_qk(const QkNormRope& a, QkGrid grid, bool backward, bool interleaved, hipStream_t st) {
  auto kernel = backward ? (interleaved ? qk_norm_rope_bwd_kernel<T, VEC, LPR, true> : qk_norm_rope_bwd_kernel<T, VEC, LPR, false>)
                         : (interleaved ? qk_norm_rope_fwd_kernel<T, VEC, LPR, true> : qk_norm_rope_fwd_kernel<T, VEC, LPR, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid.x, (unsigned)grid.y), dim3(256), 0, st, a);
  return launch_ok("norm and rotation kernel") ? SPARK_OK : SPARK_ERR_LAUNCH;
}
template <typename T>
int dispatch_qk(const QkNormRope& a, QkGrid grid, bool backward, bool interleaved, hipStream_t st) {
  if (qk_vec(a.d, a.rd) == 8)
    return a.d <= 64 ? launch_qk<T, 8, 4>(a, grid, backward, interleaved, st) : launch_qk<T, 8, 8>(a, grid, backward, interleaved, st);
  return a.d <= 64 ? launch_qk<T, 4, 8>(a, grid, backward, interleaved, st) : launch_qk<T, 4, 16>(a, grid, backward, interleaved, st);
}

}  // namespace

extern "C" {

int spark_qk_norm_rope_fwd(const void* Q, const void* K, const void* wq, const void* wk, const float* cos, const float* sin,
                           const int* positions, void* Qr, void* Kr, const spark_strides_t* sQ, const spark_strides_t* sK,
                           const spark_strides_t* sQr, const spark_strides_t* sKr, int B, int N, int H, int Hkv, int d,
                           int rd, int table, float eps, int interleaved, int w_fp32, spark_dtype_t dtype, void* stream) {
  if (!Q || !K || !Qr || !Kr || (rd > 0 && (!cos || !sin))) return SPARK_ERR_NULL;
  QkNormRope a{};
  int rc = make_qk(&a, B, N, H, Hkv, d, rd, table, eps, w_fp32, (int)dtype);
  if (rc != SPARK_OK) return rc;
  if (rd > 0 && !positions && N > table) return SPARK_ERR_SHAPE;
  if ((rc = check_rows(sQ, B, H, N, d, false, &a.mq)) != SPARK_OK) return rc;
  if ((rc = check_rows(sK, B, Hkv, N, d, false, &a.mk)) != SPARK_OK) return rc;
  if ((rc = check_rows(sQr, B, H, N, d, true, &a.moq)) != SPARK_OK) return rc;
  if ((rc = check_rows(sKr, B, Hkv, N, d, true, &a.mok)) != SPARK_OK) return rc;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Qr) || !aligned16(Kr) || !aligned16(cos) || !aligned16(sin))
    return SPARK_ERR_ALIGN;
  a.q = Q; a.k = K; a.oq = Qr; a.ok = Kr; a.wq = wq; a.wk = wk; a.cos = cos; a.sin = sin; a.positions = positions;
  const QkGrid grid = qk_grid(&a, false);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == SPARK_F16 ? dispatch_qk<_Float16>(a, grid, false, interleaved != 0, st)
                            : dispatch_qk<__bf16>(a, grid, false, interleaved != 0, st);
}

size_t spark_qk_norm_rope_bwd_workspace_bytes(int B, int N, int H, int Hkv, int d, int rd, spark_dtype_t dtype) {
  QkNormRope a{};
  if (make_qk(&a, B, N, H, Hkv, d, rd, 1, 1.0f, 0, (int)dtype) != SPARK_OK) return 0;
  const QkGrid grid = qk_grid(&a, true);
  return (size_t)grid.x * (size_t)grid.y * (size_t)d * sizeof(float);
}

int spark_qk_norm_rope_bwd(const void* Q, const void* K, const void* wq, const void* wk, const float* cos, const float* sin,
                           const int* positions, const void* dQr, const void* dKr, void* dQ, void* dK, float* dwq,
                           float* dwk, const spark_strides_t* sQ, const spark_strides_t* sK, const spark_strides_t* sdQr,
                           const spark_strides_t* sdKr, const spark_strides_t* sdQ, const spark_strides_t* sdK,
                           void* workspace, size_t workspace_bytes, int B, int N, int H, int Hkv, int d, int rd, int table,
                           float eps, int interleaved, int w_fp32, spark_dtype_t dtype, void* stream) {
  if (!Q || !K || !dQr || !dKr || !dQ || !dK || !dwq || !dwk || !workspace || (rd > 0 && (!cos || !sin)))
    return SPARK_ERR_NULL;
  QkNormRope a{};
  int rc = make_qk(&a, B, N, H, Hkv, d, rd, table, eps, w_fp32, (int)dtype);
  if (rc != SPARK_OK) return rc;
  if (rd > 0 && !positions && N > table) return SPARK_ERR_SHAPE;
  if ((rc = check_rows(sQ, B, H, N, d, false, &a.mq)) != SPARK_OK) return rc;
  if ((rc = check_rows(sK, B, Hkv, N, d, false, &a.mk)) != SPARK_OK) return rc;
  if ((rc = check_rows(sdQr, B, H, N, d, false, &a.mgq)) != SPARK_OK) return rc;
  if ((rc = check_rows(sdKr, B, Hkv, N, d, false, &a.mgk)) != SPARK_OK) return rc;
  if ((rc = check_rows(sdQ, B, H, N, d, true, &a.moq)) != SPARK_OK) return rc;
  if ((rc = check_rows(sdK, B, Hkv, N, d, true, &a.mok)) != SPARK_OK) return rc;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(dQr) || !aligned16(dKr) || !aligned16(dQ) || !aligned16(dK) ||
      !aligned16(cos) || !aligned16(sin) || !aligned16(workspace))
    return SPARK_ERR_ALIGN;
  const QkGrid grid = qk_grid(&a, true);
  const int parts = grid.x * grid.y;
  if (workspace_bytes < (size_t)parts * (size_t)d * sizeof(float)) return SPARK_ERR_WORKSPACE;
  a.q = Q; a.k = K; a.dq_out = dQr; a.dk_out = dKr; a.oq = dQ; a.ok = dK; a.wq = wq; a.wk = wk; a.cos = cos; a.sin = sin;
  a.positions = positions;
  a.partial = static_cast<float*>(workspace);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  rc = dtype == SPARK_F16 ? dispatch_qk<_Float16>(a, grid, true, interleaved != 0, st)
                          : dispatch_qk<__bf16>(a, grid, true, interleaved != 0, st);
  if (rc != SPARK_OK) return rc;
  hipLaunchKernelGGL(qk_norm_dw_kernel, dim3((unsigned)((d + 15) / 16), 2), dim3(1024), 0, st, a.partial, dwq, dwk, d,
                     grid.x * a.q_groups, parts);
  return launch_ok("weight gradient kernel") ? SPARK_OK : SPARK_ERR_LAUNCH;
}

}  // extern "C"
