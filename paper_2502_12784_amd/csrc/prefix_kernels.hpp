// Attention of a batch whose sequences come in groups that share a prefix: sequence b of group b / (B / G) attends to the
// group's prefix (keys and values [G,Hkv,P,d], there once) and then to its own suffix ([B,Hkv,S,d]).
//
// Softmax over the keys of both parts has one maximum and one sum, so a query tile walks the tiles of the prefix and then
// those of its suffix in the forward's loop (fwd_kernel.hpp): nothing is merged, and nothing is written but O and LSE.
#pragma once
#include "fwd_kernel.hpp"

namespace spark {

struct PrefixProblem {
  const void *Q, *Kp, *Vp, *Ks, *Vs;
  TensorMap mq, mkp, mvp, mks, mvs, mo;
  const int *prefix_lens, *q_lens, *s_lens;  // [G], [B], [B], or nullptr: P, Nq, S
  int G, B, H, Hkv, Nq, P, S, dh, causal;
};

// Lengths come from device memory: whatever stands there, no tensor is read or written beyond its size.
static __device__ __forceinline__ int length_of(const int* lens, int i, int most) {
  if (!lens) return most;
  const int n = lens[i];
  return n < 0 ? 0 : n < most ? n : most;
}

// A query ahead that hides no suffix key: less than 2^31 with any row index (below 2^27) added.
constexpr int ALL_AHEAD = 1 << 30;

// What one (sequence, head) attends to.  `flat` orders them by prefix and head of keys, so that those that share keys are
// neighbours and run on the same XCD.
struct PrefixHead {
  int b, h, hk, grp;
  int P, rows, S, ahead;
  __device__ __forceinline__ PrefixHead(const PrefixProblem& p, int flat) {
    const int per = p.H / p.Hkv, seqs = p.B / p.G;
    const int sub = flat % (seqs * per);
    flat /= seqs * per;
    hk = flat % p.Hkv;
    grp = flat / p.Hkv;
    b = grp * seqs + sub / per;
    h = hk * per + sub % per;
    P = length_of(p.prefix_lens, grp, p.P);
    rows = length_of(p.q_lens, b, p.Nq);
    S = length_of(p.s_lens, b, p.S);
    ahead = p.causal ? S - rows : ALL_AHEAD;
  }
};
template <typename T>
static __device__ __forceinline__ const T* head_of(const void* x, const TensorMap& m, int outer, int head) {
  return static_cast<const T*>(x) + (size_t)outer * (size_t)m.batch + (size_t)head * (size_t)m.head;
}
static __device__ __forceinline__ uint32_t span_or_none(const TensorMap& m, int n, int dh) {
  return n ? head_span_bytes(m, n, dh) : 0;
}

// Rows [row0, row1) of one head of an output, all zeros, by the whole workgroup.
template <typename T>
static __device__ __forceinline__ void zero_rows(T* head, const TensorMap& m, int row0, int row1, int dh) {
  const int chunks = dh / 8;
  for (int i = threadIdx.x; i < (row1 - row0) * chunks; i += blockDim.x) {
    const int r = i / chunks;
    *reinterpret_cast<u32x4*>(head + (size_t)(row0 + r) * (size_t)m.row + (i - r * chunks) * 8) = u32x4{0, 0, 0, 0};
  }
}

template <typename T, int D, int NW, bool PAIR>
__global__ __launch_bounds__(64 * NW, NW == 4 ? (D == 64 ? 3 : 2) : 1) void mha_prefix_fwd_kernel(
    PrefixProblem p, T* __restrict__ O, float* __restrict__ LSE, int nqt, float scale_log2) {
  const int logical = xcd_contiguous(blockIdx.x, gridDim.x);
  const int flat = logical / nqt, item = logical - flat * nqt;
  const PrefixHead x(p, flat);
  const int head = x.b * p.H + x.h;
  constexpr int BM = FwdCfg<D, NW, PAIR>::BM;
  // the causal loop takes the tiles from the last (longest) one on
  const int row0 = (nqt - 1 - item) * BM, row1 = row0 + BM < p.Nq ? row0 + BM : p.Nq;
  if (row0 >= x.rows || (x.P == 0 && (x.S == 0 || row1 + x.ahead <= 0))) {  // no row in use, or no key for any
    zero_rows(O + (size_t)x.b * (size_t)p.mo.batch + (size_t)x.h * (size_t)p.mo.head, p.mo, row0, row1, p.dh);
    for (int i = row0 + threadIdx.x; i < row1; i += 64 * NW) LSE[(size_t)head * p.Nq + i] = -INFINITY;
    return;
  }
  PrefixAndSuffix<T> keys;
  keys.head = head;
  keys.item = item;
  keys.Kp = head_of<T>(p.Kp, p.mkp, x.grp, x.hk);
  keys.Vp = head_of<T>(p.Vp, p.mvp, x.grp, x.hk);
  keys.kp_row_bytes = (uint32_t)p.mkp.row * 2;
  keys.vp_row_bytes = (uint32_t)p.mvp.row * 2;
  keys.kp_bytes = span_or_none(p.mkp, x.P, p.dh);
  keys.vp_bytes = span_or_none(p.mvp, x.P, p.dh);
  keys.P = x.P;
  keys.rows = x.rows;
  keys.ahead = x.ahead;
  fwd_tiles<T, D, true, false, NW, PAIR>(static_cast<const T*>(p.Q), head_of<T>(p.Ks, p.mks, x.b, x.hk),
                                         head_of<T>(p.Vs, p.mvs, x.b, x.hk), O, LSE, p.mq, p.mks, p.mvs, p.mo, p.H, p.Nq,
                                         x.S, p.dh, nqt, 0, scale_log2, Dropout{}, keys);
}

}  // namespace spark
