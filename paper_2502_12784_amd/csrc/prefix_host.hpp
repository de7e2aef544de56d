// Host side of spark_mha_prefix_*: argument checks, launch shapes, dispatch.
#pragma once
#include "host_util.hpp"
#include "prefix_kernels.hpp"

namespace {

// A tensor [outer, heads, n, d] of the operator, n >= 0.  The stride of an index with one value does not matter.  The
// kernels address a head through 32-bit offsets, as in check_strides.
int check_part(const void* x, const spark_strides_t* s, int outer, int heads, int n, int d, bool is_output, TensorMap* out) {
  if (!s || (!x && n > 0)) return SPARK_ERR_NULL;
  const TensorMap m{outer > 1 ? s->batch : 0, heads > 1 ? s->head : 0, n > 1 ? s->row : d};
  if (m.batch < 0 || m.head < 0 || m.row < d) return SPARK_ERR_SHAPE;
  if (is_output && n > 0 && ((outer > 1 && m.batch == 0) || (heads > 1 && m.head == 0))) return SPARK_ERR_SHAPE;
  if ((m.batch | m.head | m.row) & 7) return SPARK_ERR_ALIGN;
  if (m.row >= (int64_t)1 << 30 || (int64_t)(n + 256) * m.row * 2 >= (int64_t)1 << 31) return SPARK_ERR_SHAPE;
  if (!aligned16(x)) return SPARK_ERR_ALIGN;
  *out = m;
  return SPARK_OK;
}

// Sizes and flags.  Products that later become grid sizes or element counts are bounded here.
int make_prefix(PrefixProblem* p, int G, int B, int H, int Hkv, int Nq, int P, int S, int d, float scale, int causal, int dtype) {
  if (dtype != SPARK_F16 && dtype != SPARK_BF16) return SPARK_ERR_DTYPE;
  if (G < 1 || B < 1 || H < 1 || Hkv < 1 || Nq < 1 || P < 0 || S < 0 || (P == 0 && S == 0)) return SPARK_ERR_SHAPE;
  if (B % G || H % Hkv || d < 8 || d > 128 || (d & 7)) return SPARK_ERR_SHAPE;
  if (!isfinite(scale) || !(scale > 0.f)) return SPARK_ERR_SHAPE;
  const int64_t n = Nq > P ? (Nq > S ? Nq : S) : (P > S ? P : S);
  if ((n + 256) * d * 2 >= (int64_t)1 << 31) return SPARK_ERR_SHAPE;
  if ((int64_t)B * H >= (int64_t)1 << 24 || (int64_t)B * H * ((n + 31) / 32) >= (int64_t)1 << 31) return SPARK_ERR_SHAPE;
  p->G = G; p->B = B; p->H = H; p->Hkv = Hkv; p->Nq = Nq; p->P = P; p->S = S; p->dh = d; p->causal = causal != 0;
  return SPARK_OK;
}

template <typename T, int D, int NW, bool PAIR>
int launch_prefix_fwd(const PrefixProblem& p, void* O, float* LSE, float scale, hipStream_t st) {
  using C = FwdCfg<D, NW, PAIR>;
  auto kernel = mha_prefix_fwd_kernel<T, D, NW, PAIR>;
  static std::atomic<uint64_t> ready{0};
  const int attr = ensure_smem(kernel, C::SMEM, ready);
  if (attr != SPARK_OK) return attr;
  const int nqt = (p.Nq + C::BM - 1) / C::BM;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.B * p.H * nqt)), dim3(64 * NW), C::SMEM, st, p, static_cast<T*>(O), LSE, nqt,
                     scale * 1.4426950408889634f);
  return launch_ok("forward kernel (prefix)") ? SPARK_OK : SPARK_ERR_LAUNCH;
}

template <typename T>
int dispatch_prefix_fwd(const PrefixProblem& p, void* O, float* LSE, float scale, hipStream_t st) {
  if (p.dh <= 64) return launch_prefix_fwd<T, 64, 4, false>(p, O, LSE, scale, st);
  if (p.dh <= 96) return launch_prefix_fwd<T, 96, 4, false>(p, O, LSE, scale, st);
  return launch_prefix_fwd<T, 128, 4, false>(p, O, LSE, scale, st);
}

}  // namespace

extern "C" {

size_t spark_mha_prefix_fwd_workspace_bytes(int G, int B, int H, int Hkv, int Nq, int P, int S, int d, spark_dtype_t dtype) {
  PrefixProblem p{};
  if (make_prefix(&p, G, B, H, Hkv, Nq, P, S, d, 1.0f, 0, (int)dtype) != SPARK_OK) return 0;
  return 0;
}

int spark_mha_prefix_fwd(const void* Q, const void* Kp, const void* Vp, const void* Ks, const void* Vs, void* O, float* LSE,
                         const spark_strides_t* sQ, const spark_strides_t* sKp, const spark_strides_t* sVp,
                         const spark_strides_t* sKs, const spark_strides_t* sVs, const spark_strides_t* sO,
                         const int* prefix_lens, const int* q_lens, const int* s_lens, void* workspace,
                         size_t workspace_bytes, int G, int B, int H, int Hkv, int Nq, int P, int S, int d, float scale,
                         int causal, spark_dtype_t dtype, void* stream) {
  if (!Q || !O || !LSE) return SPARK_ERR_NULL;
  PrefixProblem p{};
  int rc = make_prefix(&p, G, B, H, Hkv, Nq, P, S, d, scale, causal, (int)dtype);
  if (rc != SPARK_OK) return rc;
  if ((rc = check_part(Q, sQ, B, H, Nq, d, false, &p.mq)) != SPARK_OK) return rc;
  if ((rc = check_part(Kp, sKp, G, Hkv, P, d, false, &p.mkp)) != SPARK_OK) return rc;
  if ((rc = check_part(Vp, sVp, G, Hkv, P, d, false, &p.mvp)) != SPARK_OK) return rc;
  if ((rc = check_part(Ks, sKs, B, Hkv, S, d, false, &p.mks)) != SPARK_OK) return rc;
  if ((rc = check_part(Vs, sVs, B, Hkv, S, d, false, &p.mvs)) != SPARK_OK) return rc;
  if ((rc = check_part(O, sO, B, H, Nq, d, true, &p.mo)) != SPARK_OK) return rc;
  if (!aligned16(LSE) || !aligned16(workspace)) return SPARK_ERR_ALIGN;
  p.Q = Q; p.Kp = Kp; p.Vp = Vp; p.Ks = Ks; p.Vs = Vs;
  p.prefix_lens = prefix_lens; p.q_lens = q_lens; p.s_lens = s_lens;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == SPARK_F16 ? dispatch_prefix_fwd<_Float16>(p, O, LSE, scale, st)
                            : dispatch_prefix_fwd<__bf16>(p, O, LSE, scale, st);
}

}  // extern "C"
