// Norm of every head's query and key vector and its rotation by position, in one pass, forward and backward:
// the step between a decoder's projection and its attention.
//
//   forward    r = 1 / sqrt(mean(x^2) + eps),  n = x r,  y = n w,  out = R y
//   backward   dy = R^T dout,  dw = sum over rows of dy n,  t = dy w,  dx = r (t - n mean(t n))
//
// R turns the pairs of the first `rd` elements of a row by the angles of the row's position: (cos, sin) of pair p
// come from row `position` of two tables.  Pairs are (p, p + rd/2), or (2p, 2p + 1) if interleaved.  All of it is
// fp32; the results are rounded once.
//
// Memory-bound: the forward reads x and writes out (4 bytes an element), the backward reads x and dout and writes
// dx (6 bytes); the tables, read once per token and group of heads, and the weights add little.
//
// A lane holds both elements of its VEC pairs as two chunks of VEC elements, so that the rotation needs no other
// lane; LPR lanes hold a row and sum its squares with DPP moves.  A workgroup takes 256 / LPR tokens and one group of
// heads, walking the heads with its tokens' cos, sin and its weights in registers: read per (token, head) instead, the
// tables would be twice the traffic of x in the first-level cache.  Measured, against 5.0 TB/s of a 1 GiB copy: forward, 4 x 2048
// tokens, 16 + 16 heads of 128 26.4 us (5.1 TB/s); 16384 tokens, 32 + 8 heads of 64 forward 26.8 us (6.2 TB/s: caches hold a part),
// backward 45.9 us (5.5 TB/s).
#pragma once
#include "mma_gfx950.hpp"
#include "tiles_gfx950.hpp"

namespace spark {

struct QkNormRope {
  const void *q, *k;    // [B,H,N,d], [B,Hkv,N,d]
  const void *dq_out, *dk_out;  // backward: gradients of the results, as q and k
  void *oq, *ok;        // results, or (backward) gradients of q and k
  TensorMap mq, mk, mgq, mgk, moq, mok;
  const void *wq, *wk;  // [d], fp32 or the tensors' type; nullptr: ones
  const float *cos, *sin;  // [table, rd / 2]
  const int* positions;    // [B,N], or nullptr: the token's index
  float* partial;       // backward: a row of d sums for every workgroup
  int tokens, N, H, Hkv, d, rd, table, w_is_fp32;
  int group, q_groups;  // heads per workgroup; groups of query heads, those of key heads follow
  float eps, inv_d;
};

// Sum over LPR neighbouring lanes, LPR = 4, 8 or 16, in all of them.
template <int LPR>
static __device__ __forceinline__ float sum_lanes(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value,
                                                                 0xF, 0xF, true));
  };
  x += dpp(x, std::integral_constant<int, 0xB1>{});  // quad_perm [1,0,3,2]
  x += dpp(x, std::integral_constant<int, 0x4E>{});  // quad_perm [2,3,0,1]
  if (LPR >= 8) x += dpp(x, std::integral_constant<int, 0x141>{});   // row_half_mirror: the other quad of eight
  if (LPR >= 16) x += dpp(x, std::integral_constant<int, 0x140>{});  // row_mirror: the other eight
  return x;
}

// What a lane holds of a token: the columns of its two chunks, and its pairs' cos and sin (1, 0 behind column rd).
template <int VEC, bool INTERLEAVED> struct QkLane {
  int lo, hi;
  bool live;      // holds elements of a row that exists
  bool skip;      // padding: a negative position
  float c[VEC], s[VEC];
  size_t b, n;

  __device__ __forceinline__ QkLane(const QkNormRope& a, int j) {
    const int turned = a.rd / (2 * VEC);  // chunks of pairs that turn
    if (j < turned && !INTERLEAVED) {
      lo = j * VEC;
      hi = lo + a.rd / 2;
    } else {
      lo = 2 * j * VEC;
      hi = lo + VEC;
    }
  }
  __device__ __forceinline__ void token(const QkNormRope& a, int t, int j) {
    live = t < a.tokens && 2 * j * VEC < a.d;
    t = t < a.tokens ? t : a.tokens - 1;
    b = (unsigned)t / (unsigned)a.N;
    n = (unsigned)t - (unsigned)b * (unsigned)a.N;
    const int pos = a.positions ? a.positions[t] : (int)n;
    skip = pos < 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
    }
    if (j < a.rd / (2 * VEC) && !skip) {
      if (pos < a.table) {
        const size_t at = (size_t)pos * (size_t)(a.rd / 2) + (size_t)(j * VEC);
#pragma unroll
        for (int x = 0; x < VEC / 4; ++x) {
          const f32x4 cv = *reinterpret_cast<const f32x4*>(a.cos + at + 4 * x);
          const f32x4 sv = *reinterpret_cast<const f32x4*>(a.sin + at + 4 * x);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c[4 * x + e] = cv[e];
            s[4 * x + e] = sv[e];
          }
        }
      } else {  // behind the table: nothing is read, and the result says so
#pragma unroll
        for (int e = 0; e < VEC; ++e) c[e] = s[e] = __builtin_nanf("");
      }
    }
  }
};

// The lane's 2 VEC elements of one row, as (first, second) of its pairs: half apart they are the chunks themselves.
template <typename T, int VEC, bool INTERLEAVED>
static __device__ __forceinline__ void qk_unpack(const T (&lo)[VEC], const T (&hi)[VEC], float (&u)[VEC],
                                                 float (&v)[VEC]) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    if (INTERLEAVED) {
      u[e] = (float)(2 * e < VEC ? lo[(2 * e) % VEC] : hi[(2 * e) % VEC]);
      v[e] = (float)(2 * e < VEC ? lo[(2 * e + 1) % VEC] : hi[(2 * e + 1) % VEC]);
    } else {
      u[e] = (float)lo[e];
      v[e] = (float)hi[e];
    }
  }
}
template <typename T, int VEC>
static __device__ __forceinline__ void qk_load(T (&x)[VEC], const T* p, bool live) {
  typedef T vec __attribute__((ext_vector_type(VEC)));
  vec z;
#pragma unroll
  for (int e = 0; e < VEC; ++e) z[e] = (T)0.f;
  if (live) z = *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = z[e];
}
// Pairs (u, v) back to the two chunks, rounded.
template <typename T, int VEC, bool INTERLEAVED>
static __device__ __forceinline__ void qk_store(T* row, int lo, int hi, const float (&u)[VEC], const float (&v)[VEC]) {
  typedef T vec __attribute__((ext_vector_type(VEC)));
  vec a, b;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    if (INTERLEAVED) {
      a[e] = (T)(e & 1 ? v[e / 2] : u[e / 2]);
      b[e] = (T)(e & 1 ? v[(VEC + e) / 2] : u[(VEC + e) / 2]);
    } else {
      a[e] = (T)u[e];
      b[e] = (T)v[e];
    }
  }
  *reinterpret_cast<vec*>(row + lo) = a;
  *reinterpret_cast<vec*>(row + hi) = b;
}
// The weights of the lane's pairs.
template <typename T, int VEC, bool INTERLEAVED>
static __device__ __forceinline__ void qk_weights(const void* w, bool fp32, int lo, int hi, bool live, float (&u)[VEC],
                                                  float (&v)[VEC]) {
  float a[VEC], b[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    a[e] = b[e] = 1.f;
    if (w && live) {
      a[e] = fp32 ? static_cast<const float*>(w)[lo + e] : (float)static_cast<const T*>(w)[lo + e];
      b[e] = fp32 ? static_cast<const float*>(w)[hi + e] : (float)static_cast<const T*>(w)[hi + e];
    }
  }
  qk_unpack<float, VEC, INTERLEAVED>(a, b, u, v);
}

// Heads of a workgroup whose rows are requested together.
constexpr int QK_AHEAD = 4;

template <typename T, int VEC, int LPR, bool INTERLEAVED>
__global__ __launch_bounds__(256) void qk_norm_rope_fwd_kernel(QkNormRope a) {
  const int j = threadIdx.x % LPR;
  const bool q_side = (int)blockIdx.y < a.q_groups;
  const int g = q_side ? blockIdx.y : (int)blockIdx.y - a.q_groups, heads = q_side ? a.H : a.Hkv;
  const int h0 = g * a.group, h1 = h0 + a.group < heads ? h0 + a.group : heads;
  const TensorMap mx = q_side ? a.mq : a.mk, mo = q_side ? a.moq : a.mok;
  QkLane<VEC, INTERLEAVED> l(a, j);
  l.token(a, blockIdx.x * (256 / LPR) + threadIdx.x / LPR, j);
  float wu[VEC], wv[VEC];
  qk_weights<T, VEC, INTERLEAVED>(q_side ? a.wq : a.wk, a.w_is_fp32, l.lo, l.hi, l.live, wu, wv);
  const T* x = static_cast<const T*>(q_side ? a.q : a.k) + l.b * (size_t)mx.batch + l.n * (size_t)mx.row;
  T* o = static_cast<T*>(q_side ? a.oq : a.ok) + l.b * (size_t)mo.batch + l.n * (size_t)mo.row;
  for (int h = h0; h < h1; h += QK_AHEAD) {
    T lo[QK_AHEAD][VEC], hi[QK_AHEAD][VEC];
#pragma unroll
    for (int i = 0; i < QK_AHEAD; ++i) {
      const T* p = x + (size_t)(h + i) * (size_t)mx.head;
      qk_load<T, VEC>(lo[i], p + l.lo, l.live && h + i < h1);
      qk_load<T, VEC>(hi[i], p + l.hi, l.live && h + i < h1);
    }
#pragma unroll
    for (int i = 0; i < QK_AHEAD; ++i) {
      if (h + i >= h1) break;
      float u[VEC], v[VEC], ss = 0.f;
      qk_unpack<T, VEC, INTERLEAVED>(lo[i], hi[i], u, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) ss += u[e] * u[e] + v[e] * v[e];
      const float r = rsqrtf(sum_lanes<LPR>(ss) * a.inv_d + a.eps);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float y = u[e] * r * wu[e], z = v[e] * r * wv[e];
        u[e] = l.skip ? 0.f : y * l.c[e] - z * l.s[e];
        v[e] = l.skip ? 0.f : z * l.c[e] + y * l.s[e];
      }
      if (l.live) qk_store<T, VEC, INTERLEAVED>(o + (size_t)(h + i) * (size_t)mo.head, l.lo, l.hi, u, v);
    }
  }
}

// Gradients of the rows; the sums for dw of the workgroup's rows go to its row of `partial`, first those of the query
// heads' workgroups (blockIdx.y * gridDim.x + blockIdx.x).
template <typename T, int VEC, int LPR, bool INTERLEAVED>
__global__ __launch_bounds__(256) void qk_norm_rope_bwd_kernel(QkNormRope a) {
  __shared__ float sums[4][2 * VEC * LPR];
  const int j = threadIdx.x % LPR;
  const bool q_side = (int)blockIdx.y < a.q_groups;
  const int g = q_side ? blockIdx.y : (int)blockIdx.y - a.q_groups, heads = q_side ? a.H : a.Hkv;
  const int h0 = g * a.group, h1 = h0 + a.group < heads ? h0 + a.group : heads;
  const TensorMap mx = q_side ? a.mq : a.mk, mg = q_side ? a.mgq : a.mgk, mo = q_side ? a.moq : a.mok;
  QkLane<VEC, INTERLEAVED> l(a, j);
  float wu[VEC], wv[VEC], du[VEC], dv[VEC];
  qk_weights<T, VEC, INTERLEAVED>(q_side ? a.wq : a.wk, a.w_is_fp32, l.lo, l.hi, 2 * j * VEC < a.d, wu, wv);
#pragma unroll
  for (int e = 0; e < VEC; ++e) du[e] = dv[e] = 0.f;
  constexpr int AHEAD = QK_AHEAD / 2;  // twice the rows of the forward
  for (int t = blockIdx.x * (256 / LPR); t < a.tokens; t += gridDim.x * (256 / LPR)) {
    l.token(a, t + threadIdx.x / LPR, j);
    const T* x = static_cast<const T*>(q_side ? a.q : a.k) + l.b * (size_t)mx.batch + l.n * (size_t)mx.row;
    const T* dout = static_cast<const T*>(q_side ? a.dq_out : a.dk_out) + l.b * (size_t)mg.batch + l.n * (size_t)mg.row;
    T* o = static_cast<T*>(q_side ? a.oq : a.ok) + l.b * (size_t)mo.batch + l.n * (size_t)mo.row;
    for (int h = h0; h < h1; h += AHEAD) {
      T xlo[AHEAD][VEC], xhi[AHEAD][VEC], glo[AHEAD][VEC], ghi[AHEAD][VEC];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const T* p = x + (size_t)(h + i) * (size_t)mx.head;
        const T* q = dout + (size_t)(h + i) * (size_t)mg.head;
        const bool live = l.live && !l.skip && h + i < h1;
        qk_load<T, VEC>(xlo[i], p + l.lo, live);
        qk_load<T, VEC>(xhi[i], p + l.hi, live);
        qk_load<T, VEC>(glo[i], q + l.lo, live);
        qk_load<T, VEC>(ghi[i], q + l.hi, live);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (h + i >= h1) break;
        float u[VEC], v[VEC], gu[VEC], gv[VEC], ss = 0.f, tn = 0.f;
        qk_unpack<T, VEC, INTERLEAVED>(xlo[i], xhi[i], u, v);
        qk_unpack<T, VEC, INTERLEAVED>(glo[i], ghi[i], gu, gv);
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss += u[e] * u[e] + v[e] * v[e];
        const float r = rsqrtf(sum_lanes<LPR>(ss) * a.inv_d + a.eps);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float yu = gu[e] * l.c[e] + gv[e] * l.s[e], yv = gv[e] * l.c[e] - gu[e] * l.s[e];
          u[e] *= r;
          v[e] *= r;
          du[e] += yu * u[e];
          dv[e] += yv * v[e];
          gu[e] = yu * wu[e];
          gv[e] = yv * wv[e];
          tn += gu[e] * u[e] + gv[e] * v[e];
        }
        const float m = sum_lanes<LPR>(tn) * a.inv_d;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          gu[e] = r * (gu[e] - u[e] * m);
          gv[e] = r * (gv[e] - v[e] * m);
        }
        if (l.live) qk_store<T, VEC, INTERLEAVED>(o + (size_t)(h + i) * (size_t)mo.head, l.lo, l.hi, gu, gv);
      }
    }
  }
  // over the wave's tokens, then over the waves
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
#pragma unroll
    for (int m = LPR; m < 64; m <<= 1) {
      du[e] += __shfl_xor(du[e], m);
      dv[e] += __shfl_xor(dv[e], m);
    }
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (lane < LPR) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      sums[wave][j * 2 * VEC + e] = du[e];
      sums[wave][j * 2 * VEC + VEC + e] = dv[e];
    }
  }
  __syncthreads();
  const int part = blockIdx.y * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < a.d; i += 256) {
    // column of entry i of the lanes' sums: lane i / (2 VEC), its u's, then its v's
    const int lane_j = i / (2 * VEC), e = i % VEC, second = i / VEC & 1;
    int col;
    if (lane_j < a.rd / (2 * VEC) && !INTERLEAVED)
      col = lane_j * VEC + e + second * (a.rd / 2);
    else
      col = INTERLEAVED ? lane_j * 2 * VEC + 2 * e + second : lane_j * 2 * VEC + second * VEC + e;
    a.partial[(size_t)part * (size_t)a.d + col] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
  }
}

// dw of one side from the partial sums, in their order: 16 columns to a workgroup, 64 sums of every column side by side: one round
// trip to memory for 1024 rows (500 of 80 columns 3.0 ... 3.8 us, 768 of 64 4.6).
__global__ __launch_bounds__(1024) void qk_norm_dw_kernel(const float* __restrict__ partial, float* __restrict__ dwq,
                                                          float* __restrict__ dwk, int d, int q_parts, int parts) {
  __shared__ float sums[64][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  const int first = blockIdx.y == 0 ? 0 : q_parts, last = blockIdx.y == 0 ? q_parts : parts;
  float acc = 0.f;
  if (col < d) {
    for (int p = first + r; p < last; p += 16 * 64) {  // sixteen requested together
      float x[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u] = p + u * 64 < last ? partial[(size_t)(p + u * 64) * (size_t)d + col] : 0.f;
#pragma unroll
      for (int u = 0; u < 16; ++u) acc += x[u];
    }
  }
  sums[r][c] = acc;
  __syncthreads();
  if (r == 0 && col < d) {
    acc = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) acc += sums[i][c];
    (blockIdx.y == 0 ? dwq : dwk)[col] = acc;
  }
}

}  // namespace spark
