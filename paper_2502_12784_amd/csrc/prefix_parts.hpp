// Attention behind a shared prefix for few query rows per sequence (a new token, some drafted ones) or few workgroups.
//
// One query row per head leaves 31 of a wave's 32 matrix columns empty, and every sequence would read the prefix by itself.
// Here the rows of all sequences and query heads that share a head of the prefix are packed into common tiles, so the prefix
// is read (and multiplied) once per tile: 64 sequences with four query heads to a head of keys make two tiles of 128 rows.
// Runs of keys go to different workgroups, and every row's results over the runs are merged at the end (Eq. 3):
//   * runs of the prefix against tiles of 128 packed rows, in the forward's loop (fwd_tiles, four waves share the K/V tiles):
//     with many rows this is a matrix product; up to 32 rows in the split forward's loop, which is a read of K and V;
//   * runs of a sequence's suffix against its own packed rows (heads, queries), 32 to a tile, four waves with a stream of
//     keys each (fwd_split_tiles): a read of K and V;
//   * mha_prefix_merge_kernel adds a row's partial results, as many of them requested at once as there are lanes for.
// Both kinds of runs are in one grid, two workgroups to a CU: the products of the prefix overlap with the reads of the
// suffixes.  A partial result is lds_row<D> + 4 floats: O, unnormalised, m, l (0: the run had no key for the row).
//
// Bound by memory, and for the smaller ones by the latency of two kernels.  Measured, one new token, d = 128, bf16: 32 sequences x 16
// heads behind 4096 + up to 256 keys 18.6 us (4.6 TB/s; a read of 1 GiB reaches 4.0, a copy 5.0) and 4.0 for the merge; 64 x 32 heads over 8 behind
// 16384 + up to 512 35.5 (4.7 TB/s, and 17.6 GFLOP) and 5.6.
#pragma once
#include "fwd_split_kernel.hpp"
#include "prefix_kernels.hpp"

namespace spark {

struct PrefixParts {
  float* partial;       // [rows][p_parts + s_parts][lds_row<D> + 4], rows = (b * H + h) * Nq + i
  int p_parts, s_parts; // runs of a prefix, of a suffix
  int p_tiles, s_tiles; // tiles of rows of a prefix, of a suffix
  int p_items;          // workgroups of the prefix, in front of those of the suffixes
  int wide;             // tiles of 128 rows for the prefix, or of 32
};

// Row `r` of the `n` packed rows (sequence b0 + r / (Nq per), query, query head) of head hk of the keys.
template <typename T>
static __device__ __forceinline__ int pack_row(const PrefixProblem& p, const PrefixParts& s, int b0, int hk, int r, int n,
                                               int part, int width, PackedRows<T>* out) {
  const int per = p.H / p.Hkv, each = p.Nq * per;
  const bool there = r < n;
  const int at = there ? r : 0;
  const int b = b0 + at / each, rest = at % each, i = rest / per, h = hk * per + rest % per;
  out->q = head_of<T>(p.Q, p.mq, b, h) + (size_t)i * (size_t)p.mq.row;
  const bool used = there && i < length_of(p.q_lens, b, p.Nq);
  const size_t row = ((size_t)b * p.H + h) * (size_t)p.Nq + (size_t)i;
  out->out = used ? s.partial + (row * (size_t)(s.p_parts + s.s_parts) + (size_t)part) * (size_t)(width + 4) : nullptr;
  return i;
}

template <typename T>
static __device__ __forceinline__ const T* uniform(const T* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  // the builtin returns an int: without the conversion the lower half would fill the upper one with its sign
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)a), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32));
  return reinterpret_cast<const T*>((uint64_t)hi << 32 | lo);
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void mha_prefix_parts_kernel(PrefixProblem p, PrefixParts s, float scale_log2) {
  constexpr int W = lds_row<D>;
  using Narrow = FwdSplitCfg<W, 4>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.H / p.Hkv;
  const TensorMap none{0, 0, 0};
  PackedRows<T> rows;
  rows.item = 0;
  // the run: keys [k0, k0 + n) of a prefix or suffix with `all` keys, `run` to a part
  int hk, part, k0, n;
  const T *K, *V;
  TensorMap mk, mv;
  bool wide = false;
  if ((int)blockIdx.x < s.p_items) {
    const int logical = xcd_contiguous(blockIdx.x, s.p_items);
    const int tile = logical % s.p_tiles, unit = logical / s.p_tiles;
    part = unit % s.p_parts;
    const int owner = unit / s.p_parts, grp = owner / p.Hkv, seqs = p.B / p.G;
    hk = owner - grp * p.Hkv;
    wide = s.wide;
    const int bn = wide ? FwdCfg<D>::BN : Narrow::BN, all = length_of(p.prefix_lens, grp, p.P);
    const int run = ((all + bn - 1) / bn + s.p_parts - 1) / s.p_parts * bn;
    k0 = part * run;
    n = all - k0 < run ? all - k0 : run;
    const int r = wide ? tile * 128 + wave * 32 + (lane & 31) : tile * 32 + (lane & 31);
    pack_row(p, s, grp * seqs, hk, r, seqs * p.Nq * per, part, W, &rows);
    rows.seen = rows.seen_by_all = n;
    K = head_of<T>(p.Kp, p.mkp, grp, hk);
    V = head_of<T>(p.Vp, p.mvp, grp, hk);
    mk = p.mkp;
    mv = p.mvp;
  } else {
    const int logical = xcd_contiguous(blockIdx.x - s.p_items, gridDim.x - s.p_items);
    const int tile = logical % s.s_tiles, unit = logical / s.s_tiles;
    part = unit % s.s_parts;
    const int owner = unit / s.s_parts, b = owner / p.Hkv;
    hk = owner - b * p.Hkv;
    const int all = length_of(p.s_lens, b, p.S), q = length_of(p.q_lens, b, p.Nq), ahead = p.causal ? all - q : ALL_AHEAD;
    const int run = ((all + Narrow::BN - 1) / Narrow::BN + s.s_parts - 1) / s.s_parts * Narrow::BN;
    k0 = part * run;
    n = all - k0 < run ? all - k0 : run;
    const int i = pack_row(p, s, b, hk, tile * 32 + (lane & 31), p.Nq * per, s.p_parts + part, W, &rows);
    // queries ascend with the packed rows: the tile's first sees fewest keys, its last most
    const int last = tile * 32 + 31 < p.Nq * per ? tile * 32 + 31 : p.Nq * per - 1;
    auto seen = [&](int query) {
      const int keys = query + ahead + 1 - k0;
      return keys < 0 ? 0 : keys < n ? keys : n;
    };
    rows.seen = seen(i);
    rows.seen_by_all = seen(tile * 32 / per);
    n = seen(last / per);
    K = head_of<T>(p.Ks, p.mks, b, hk);
    V = head_of<T>(p.Vs, p.mvs, b, hk);
    mk = p.mks;
    mv = p.mvs;
  }
  if (n <= 0) {  // nothing to attend to: the merge leaves this part out
    if (wave == 0 || wide) {
      if (lane < 32 && rows.out) *reinterpret_cast<f32x4*>(rows.out + W) = f32x4{-1e30f, 0.f, 0.f, 0.f};
    }
    return;
  }
  // Both are the same in all lanes, but the divisions on the way to them run on the vector unit; the descriptors of K and V
  // have to be in scalar registers.
  k0 = __builtin_amdgcn_readfirstlane(k0);
  n = __builtin_amdgcn_readfirstlane(n);
  K = uniform(K + (size_t)k0 * (size_t)mk.row);
  V = uniform(V + (size_t)k0 * (size_t)mv.row);
  if (wide)
    fwd_tiles<T, D, false, false, 4, false>(nullptr, K, V, nullptr, nullptr, none, mk, mv, none, 1, 1, n, p.dh, 1, 0,
                                            scale_log2, Dropout{}, rows);
  else
    fwd_split_tiles<T, W, false, false, true, 4>(nullptr, K, V, nullptr, nullptr, none, mk, mv, none, 1, 1, n, p.dh, 1, 0,
                                                 scale_log2, Dropout{}, 1, nullptr, rows);
}

// Few keys and few rows: a workgroup takes all keys of 32 packed rows of one sequence, its waves a stream each
// (fwd_split_tiles), and nothing is merged afterwards.  Bound by the latency of a chain of tiles, K and V coming from the second-level
// cache: about 1 us for every tile of each wave (4 sequences x 16 heads over 4 x 128 queries behind 1024: 13.7 us).
template <typename T, int W, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void mha_prefix_short_kernel(PrefixProblem p, T* __restrict__ O,
                                                                                    float* __restrict__ LSE, int nqt, float scale_log2) {
  const int logical = xcd_contiguous(blockIdx.x, gridDim.x);
  const int flat = logical / nqt, item = logical - flat * nqt;
  const PrefixHead x(p, flat);
  const PrefixAndSuffix<T> keys = keys_of<T>(p, x, item);
  const int h0 = x.hk * keys.per, all = p.Nq * keys.per;
  O += (size_t)x.b * (size_t)p.mo.batch + (size_t)h0 * (size_t)p.mo.head;
  LSE += ((size_t)x.b * p.H + h0) * (size_t)p.Nq;
  const int row0 = item * 32, row1 = row0 + 32 < all ? row0 + 32 : all;
  if (row0 >= keys.rows || (x.P == 0 && (x.S == 0 || (row1 - 1) / keys.per + x.ahead < 0))) {  // no row in use, or no key for any
    zero_rows(O, p.mo, keys, row0, row1, p.dh);
    for (int r = row0 + threadIdx.x; r < row1; r += 64 * NW) LSE[keys.stat(r)] = -INFINITY;
    return;
  }
  fwd_split_tiles<T, W, false, false, false, NW>(head_of<T>(p.Q, p.mq, x.b, h0), head_of<T>(p.Ks, p.mks, x.b, x.hk),
                                                head_of<T>(p.Vs, p.mvs, x.b, x.hk), O, LSE, p.mq, p.mks, p.mvs, p.mo, p.H, all,
                                                x.S, p.dh, nqt, 0, scale_log2, Dropout{}, 1, nullptr, keys);
}

// A row's parts: W / 4 lanes to a part, SIDE of them side by side, four requested together by each; as many rows to a
// workgroup as then fit.
template <typename T, int W, int SIDE>
__global__ __launch_bounds__(256) void mha_prefix_merge_kernel(PrefixProblem p, const float* __restrict__ partial, int parts,
                                                               T* __restrict__ O, float* __restrict__ LSE) {
  using v4 = typename Frag<T>::v4;
  constexpr int LPR = W / 4, ROWS = 256 / (LPR * SIDE);
  __shared__ float top[ROWS][SIDE];
  __shared__ f32x4 sums[ROWS][SIDE][LPR + 1];
  const int c = threadIdx.x % LPR, side = threadIdx.x / LPR % SIDE, slot = threadIdx.x / (LPR * SIDE);
  const size_t rows = (size_t)p.B * p.H * (size_t)p.Nq, row = (size_t)blockIdx.x * ROWS + slot;
  const int bh = (int)(row / (size_t)p.Nq), i = (int)(row - (size_t)bh * p.Nq), b = bh / p.H, h = bh - b * p.H;
  const bool used = row < rows && i < length_of(p.q_lens, b, p.Nq);
  const float* x = partial + row * (size_t)parts * (W + 4);
  float m = -1e30f, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (used) {
    for (int s0 = side; s0 < parts; s0 += 4 * SIDE) {
      f32x4 st[4], v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = s0 + u * SIDE;
        const float* q = x + (size_t)(s < parts ? s : s0) * (W + 4);
        st[u] = *reinterpret_cast<const f32x4*>(q + W);
        v[u] = *reinterpret_cast<const f32x4*>(q + 4 * c);
        if (s >= parts) st[u][1] = 0.f;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (st[u][1] == 0.f) continue;  // no key: O was not written
        const float m_new = fmaxf(m, st[u][0]), a = __builtin_amdgcn_exp2f(m - m_new), w = __builtin_amdgcn_exp2f(st[u][0] - m_new);
        m = m_new;
        l = l * a + st[u][1] * w;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * a + v[u][e] * w;
      }
    }
  }
  if (SIDE > 1) {
    if (c == 0) top[slot][side] = m;
    __syncthreads();
    float all = top[slot][0];
#pragma unroll
    for (int s = 1; s < SIDE; ++s) all = fmaxf(all, top[slot][s]);
    const float w = __builtin_amdgcn_exp2f(m - all);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= w;
    sums[slot][side][c] = o;
    if (c == 0) sums[slot][side][LPR][0] = l * w;
    m = all;
    __syncthreads();
    if (side) return;
    l = sums[slot][0][LPR][0];
#pragma unroll
    for (int s = 1; s < SIDE; ++s) {
      l += sums[slot][s][LPR][0];
      o += sums[slot][s][c];
    }
  }
  if (row >= rows) return;
  if (c == 0) LSE[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  if (4 * c < p.dh) {
    const float inv = 1.0f / l;
    v4 pk;
#pragma unroll
    for (int e = 0; e < 4; ++e) pk[e] = (T)(l == 0.f ? 0.f : o[e] * inv);
    *reinterpret_cast<v4*>(O + (size_t)b * (size_t)p.mo.batch + (size_t)h * (size_t)p.mo.head + (size_t)i * (size_t)p.mo.row +
                           4 * c) = pk;
  }
}

}  // namespace spark
