// Attention of a batch whose sequences come in groups that share a prefix: sequence b of group b / (B / G) attends to the
// group's prefix (keys and values [G,Hkv,P,d], there once) and then to its own suffix ([B,Hkv,S,d]).
//
// Softmax over the keys of both parts has one maximum and one sum, so a query tile walks the tiles of the prefix and then
// those of its suffix in the forward's loop (fwd_kernel.hpp): nothing is merged, and nothing is written but O and LSE.
//
// Backward.  P = exp(S - LSE) and D = rowsum(dO o O) belong to a row as a whole, so dS = P o (dP - D) can be formed part by
// part.  dQ walks both parts as the forward does.  dK and dV of a suffix tile sum over the rows of the heads that share it,
// those of a prefix tile over the rows of all sequences of the group too: the loop of bwd_dkdv_pipe, whose stages of 64 rows
// then come from one (sequence, head) after the other.  That sum is long and there are few such tiles: `parts` workgroups
// share it, and likewise a suffix tile's where the batch is small; each leaves its part in fp32, and a small kernel adds them
// in their order.
//
// Bound by the loops' instruction mixes, as in the kernels they come from.  Measured, bf16, causal, d = 128, 8 sequences x 16 heads x 1024
// queries behind 4096 + 1024 keys: forward 290 us (1.07 PFLOP/s), dQ 426 (1.09, three products), dK/dV 627 ... 660 (0.94 ... 0.99, four);
// 16 sequences x 16 heads over 4 x 257 ... 512 queries behind 1024 keys in two groups: 83, 116 and 185, and 6.6 for the sum.
#pragma once
#include "bwd_kernels.hpp"
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

// What the query heads of one (sequence, head of keys) attend to.  `flat` orders them by prefix and head of keys, so that
// those that share keys are neighbours and run on the same XCD.
struct PrefixHead {
  int b, hk, grp;
  int P, q, S, ahead;  // lengths
  __device__ __forceinline__ PrefixHead(const PrefixProblem& p, int flat) {
    const int seqs = p.B / p.G, sub = flat % seqs;
    flat /= seqs;
    hk = flat % p.Hkv;
    grp = flat / p.Hkv;
    b = grp * seqs + sub;
    P = length_of(p.prefix_lens, grp, p.P);
    q = length_of(p.q_lens, b, p.Nq);
    S = length_of(p.s_lens, b, p.S);
    ahead = p.causal ? S - q : ALL_AHEAD;
  }
};
template <typename T>
static __device__ __forceinline__ const T* head_of(const void* x, const TensorMap& m, int outer, int head) {
  return static_cast<const T*>(x) + (size_t)outer * (size_t)m.batch + (size_t)head * (size_t)m.head;
}
static __device__ __forceinline__ uint32_t span_or_none(const TensorMap& m, int n, int dh) {
  return n ? head_span_bytes(m, n, dh) : 0;
}

// Packed rows [row0, row1) of an output (`out`: of the first of their heads), all zeros, by the whole workgroup; and rows
// of one head.
template <typename T>
static __device__ __forceinline__ void zero_rows(T* out, const TensorMap& m, const PrefixAndSuffix<T>& keys, int row0, int row1,
                                                 int dh) {
  const int chunks = dh / 8;
  for (int i = threadIdx.x; i < (row1 - row0) * chunks; i += blockDim.x) {
    const int r = i / chunks;
    *reinterpret_cast<u32x4*>(out + keys.offset(m, row0 + r) + (i - r * chunks) * 8) = u32x4{0, 0, 0, 0};
  }
}
template <typename T>
static __device__ __forceinline__ void zero_rows(T* head, const TensorMap& m, int row0, int row1, int dh) {
  const int chunks = dh / 8;
  for (int i = threadIdx.x; i < (row1 - row0) * chunks; i += blockDim.x) {
    const int r = i / chunks;
    *reinterpret_cast<u32x4*>(head + (size_t)(row0 + r) * (size_t)m.row + (i - r * chunks) * 8) = u32x4{0, 0, 0, 0};
  }
}

// The keys of the workgroup's tile of packed rows.
template <typename T>
static __device__ __forceinline__ PrefixAndSuffix<T> keys_of(const PrefixProblem& p, const PrefixHead& x, int item) {
  PrefixAndSuffix<T> keys;
  keys.item = item;
  keys.per = p.H / p.Hkv;
  keys.queries = p.Nq;
  keys.Kp = head_of<T>(p.Kp, p.mkp, x.grp, x.hk);
  keys.Vp = head_of<T>(p.Vp, p.mvp, x.grp, x.hk);
  keys.kp_row_bytes = (uint32_t)p.mkp.row * 2;
  keys.vp_row_bytes = (uint32_t)p.mvp.row * 2;
  keys.kp_bytes = span_or_none(p.mkp, x.P, p.dh);
  keys.vp_bytes = span_or_none(p.mvp, x.P, p.dh);
  keys.P = x.P;
  keys.rows = x.q * keys.per;
  keys.ahead = x.ahead;
  return keys;
}

template <typename T, int D, int NW, bool PAIR>
__global__ __launch_bounds__(64 * NW, NW == 4 ? (D == 64 ? 3 : 2) : 1) void mha_prefix_fwd_kernel(
    PrefixProblem p, T* __restrict__ O, float* __restrict__ LSE, int nqt, float scale_log2) {
  const int logical = xcd_contiguous(blockIdx.x, gridDim.x);
  const int flat = logical / nqt, item = logical - flat * nqt;
  const PrefixHead x(p, flat);
  const PrefixAndSuffix<T> keys = keys_of<T>(p, x, item);
  const int h0 = x.hk * keys.per, all = p.Nq * keys.per;
  O += (size_t)x.b * (size_t)p.mo.batch + (size_t)h0 * (size_t)p.mo.head;
  LSE += ((size_t)x.b * p.H + h0) * (size_t)p.Nq;
  constexpr int BM = FwdCfg<D, NW, PAIR>::BM;
  // the causal loop takes the tiles from the last (longest) one on
  const int row0 = (nqt - 1 - item) * BM, row1 = row0 + BM < all ? row0 + BM : all;
  if (row0 >= keys.rows || (x.P == 0 && (x.S == 0 || (row1 - 1) / keys.per + x.ahead < 0))) {  // no row in use, or no key for any
    zero_rows(O, p.mo, keys, row0, row1, p.dh);
    for (int r = row0 + threadIdx.x; r < row1; r += 64 * NW) LSE[keys.stat(r)] = -INFINITY;
    return;
  }
  fwd_tiles<T, D, true, false, NW, PAIR>(head_of<T>(p.Q, p.mq, x.b, h0), head_of<T>(p.Ks, p.mks, x.b, x.hk),
                                         head_of<T>(p.Vs, p.mvs, x.b, x.hk), O, LSE, p.mq, p.mks, p.mvs, p.mo, p.H, all, x.S,
                                         p.dh, nqt, 0, scale_log2, Dropout{}, keys);
}

template <typename T> struct PrefixGrads {
  const T *dO;
  T *dQ, *dKp, *dVp, *dKs, *dVs;
  TensorMap mdo, mdq, mdkp, mdvp, mdks, mdvs;
  const float* LSE;
  float *Dws, *LSE2ws;  // [B,H,Nq]: -D, LSE * log2(e)
  float* partial;       // if parts > 1: [parts][G * Hkv][tiles of P] tiles of dK / scale and dV (PrefixTile)
  float* partial_s;     // if s_parts > 1: [s_parts][B * Hkv][tiles of S], of the suffix tiles that several workgroups share
  int parts;            // workgroups that share a prefix tile's stages evenly
  int s_parts, s_run;   // a suffix tile's stages in runs of s_run; s_parts is the most runs a tile can have
  float* partial_q;     // if q_parts > 1: [q_parts][B * Hkv][tiles of packed rows] tiles of dQ / scale, as PrefixTile but one tensor
  int q_parts;          // workgroups that share the keys of a tile of rows
};

// A part of a tile's dK / scale and dV in fp32, as the accumulators hold them: [wave][eight columns of dK, then of dV][lane][4],
// lane l with columns 4 (l / 32) + 0 ... 3 of key l % 32 of the wave: every store and load is 1 KB in one piece.  (Rows of keys
// instead, whose stores are pieces of 32 bytes: dK/dV of 16 sequences x 16 heads over 4 x 512 behind 1024 207.3 us, so 205.4.)
template <int D> struct PrefixTile {
  static constexpr int EIGHTS = 2 * D / 8, WAVE = EIGHTS * 256, FLOATS = 4 * WAVE;
  static constexpr int Q_WAVE = WAVE / 2, Q_FLOATS = FLOATS / 2;  // of dQ
};

// Of a suffix tile from key k0 on: the first block of 64 queries that sees it, and how many blocks from there on; per head.
struct SuffixBlocks {
  int first, count;
  __device__ __forceinline__ SuffixBlocks(int k0, int ahead, int queries) {
    const int row = k0 - ahead;  // the first query that sees key k0
    first = row > 0 ? row / 64 : 0;
    count = (queries + 63) / 64 - first;
    if (count < 0) count = 0;
  }
};

// The workgroup's part of dQ: `logical` counts the runs of keys of all sequences' and heads' tiles of rows.  A long prefix
// behind few rows is a long chain in few workgroups otherwise.  STATS: D and LSE * log2(e) are there already.
template <typename T, int D, bool STATS>
static __device__ __forceinline__ void prefix_dq(const PrefixProblem& p, const T* __restrict__ O, const PrefixGrads<T>& gr, int nqt,
                                                 float scale, int logical) {
  const int part = logical % gr.q_parts;
  logical /= gr.q_parts;
  const int flat = logical / nqt, item = logical - flat * nqt;
  const PrefixHead x(p, flat);
  PrefixAndSuffix<T> keys = keys_of<T>(p, x, item);
  const int h0 = x.hk * keys.per, all = p.Nq * keys.per;
  T* const dQ = gr.dQ + (size_t)x.b * (size_t)gr.mdq.batch + (size_t)h0 * (size_t)gr.mdq.head;
  const size_t stats = ((size_t)x.b * p.H + h0) * (size_t)p.Nq;
  constexpr int BM = BwdQCfg<D, true, false>::BM;
  const int row0 = (nqt - 1 - item) * BM, row1 = row0 + BM < all ? row0 + BM : all;
  if (row0 >= keys.rows || (x.P == 0 && (x.S == 0 || (row1 - 1) / keys.per + x.ahead < 0))) {  // no row in use, or no key for any
    if (part) return;
    zero_rows(dQ, gr.mdq, keys, row0, row1, p.dh);
    if (!STATS) {
      for (int r = row0 + threadIdx.x; r < row1; r += 256) {
        gr.Dws[stats + keys.stat(r)] = 0.f;
        gr.LSE2ws[stats + keys.stat(r)] = INFINITY;
      }
    }
    return;
  }
  if (gr.q_parts > 1) {
    keys.part = part;
    keys.parts = gr.q_parts;
    const size_t tiles = (size_t)p.B * (size_t)p.Hkv * (size_t)nqt, tile = ((size_t)x.b * p.Hkv + x.hk) * (size_t)nqt + (nqt - 1 - item);
    keys.sums = gr.partial_q + ((size_t)part * tiles + tile) * PrefixTile<D>::Q_FLOATS;
  }
  bwd_dq<T, D, true, false, STATS, IN_ORDER>(
      head_of<T>(p.Q, p.mq, x.b, h0), head_of<T>(p.Ks, p.mks, x.b, x.hk), head_of<T>(p.Vs, p.mvs, x.b, x.hk),
      head_of<T>(O, p.mo, x.b, h0), head_of<T>(gr.dO, gr.mdo, x.b, h0), gr.LSE + stats, gr.Dws + stats, gr.LSE2ws + stats, dQ,
      p.mq, p.mks, p.mvs, p.mo, gr.mdo, gr.mdq, p.H, all, x.S, p.dh, nqt, 0, scale, scale * 1.4426950408889634f, Dropout{}, 0,
      item, keys);
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void mha_prefix_dq_kernel(PrefixProblem p, const T* __restrict__ O, PrefixGrads<T> gr,
                                                               int nqt, float scale) {
  prefix_dq<T, D, false>(p, O, gr, nqt, scale, xcd_contiguous(blockIdx.x, gridDim.x));
}

// The query rows that see a key tile, in stages of 64 of one (sequence, head), for bwd_dkdv_pipe; and where its sums go.
template <typename T, int D> struct GroupRows {
  static constexpr bool SEVERAL = true;
  struct Stage {
    const T *q, *dout;
    const float *lse2, *dws;
    uint32_t q_bytes, do_bytes, stat_bytes;
    int block;
  };
  // of the problem, each by itself: a pointer to the kernel's arguments would put them all into scratch memory
  const T *Q, *dO;
  const float *lse2, *dws;
  const int* q_lens;
  TensorMap mq, mdo;
  int H, Nq, dh;
  int b, h;                // present pair
  int h0, h1, b_end;       // the heads that share the tile, the end of its sequences
  int left;                // stages left behind the present one, at most
  int k0;                  // causal: the tile's first key, with S keys in the suffix; -1: every row sees the tile
  int S;
  int blocks, ahead;       // of the present pair
  Stage s;
  T *dK, *dV;              // of the tile's head
  TensorMap mdk, mdv;
  int keys, all;           // keys that exist, rows that are written (zeros behind the keys)
  float* partial;          // or the workgroup's part of the tile

  __device__ __forceinline__ Stage stage() const { return s; }
  __device__ __forceinline__ int first_query() const { return s.block * 64 + ahead; }
  // Enter the present pair; whether any of its rows sees the tile.
  __device__ __forceinline__ bool enter() {
    const int rows = length_of(q_lens, b, Nq);
    ahead = k0 < 0 ? ALL_AHEAD : S - rows;
    const SuffixBlocks seen(k0, ahead, rows);
    if (!seen.count) return false;
    s.block = seen.first;
    blocks = seen.first + seen.count;
    const size_t row = ((size_t)b * H + h) * (size_t)Nq;
    s.q = head_of<T>(Q, mq, b, h);
    s.dout = head_of<T>(dO, mdo, b, h);
    s.lse2 = lse2 + row;
    s.dws = dws + row;
    s.q_bytes = head_span_bytes(mq, rows, dh);
    s.do_bytes = head_span_bytes(mdo, rows, dh);
    s.stat_bytes = (uint32_t)rows * 4;
    return true;
  }
  __device__ __forceinline__ bool next_pair() {
    for (;;) {
      if (++h == h1) {
        h = h0;
        if (++b == b_end) return false;
      }
      if (enter()) return true;
    }
  }
  // Start at stage `skip` of a suffix tile's, `each` to a head, and take `count` of them.
  __device__ __forceinline__ bool start_in(int skip, int each, int count) {
    left = count - 1;
    if (count <= 0) return false;
    h = h0 + skip / each;
    if (!enter()) return false;
    s.block += skip % each;
    return true;
  }
  __device__ __forceinline__ bool advance() {
    if (--left < 0) return false;
    if (s.block + 1 < blocks) {
      ++s.block;
      return true;
    }
    return next_pair();
  }
  // Start at stage `skip` of a prefix tile's, counted over its pairs in order, and take `count` of them.  The wave's lanes add
  // up the sequences' blocks, 64 sequences at a time.
  __device__ __forceinline__ bool start_at(int skip, int count) {
    const int per = h1 - h0, lane = threadIdx.x & 63;
    left = count - 1;
    if (count <= 0) return false;
    for (; b < b_end; b += 64) {
      int own = 0;  // stages of the lane's sequence
      if (b + lane < b_end) own = (length_of(q_lens, b + lane, Nq) + 63) / 64 * per;
      int sum = own;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int other = __shfl_up(sum, m);
        if (lane >= m) sum += other;
      }
      const uint64_t behind = __ballot(sum > skip);  // the first such sequence holds the stage
      if (behind) {
        const int at = __builtin_ctzll(behind);
        b += at;
        skip -= __builtin_amdgcn_readlane(sum - own, at);
        const int each = __builtin_amdgcn_readlane(own, at) / per;
        h = h0 + skip / each;
        if (!enter()) return false;
        s.block += skip % each;
        return true;
      }
      skip -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
  }
  // All stages of sequences [b, b_end).
  __device__ __forceinline__ int stages() const {
    const int per = h1 - h0, lane = threadIdx.x & 63;
    int own = 0;
    for (int x = b + lane; x < b_end; x += 64) own += (length_of(q_lens, x, Nq) + 63) / 64 * per;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) own += __shfl_xor(own, m);
    return __builtin_amdgcn_readfirstlane(own);
  }
  __device__ __forceinline__ void store(const f32x16 (&dk)[D / 32], const f32x16 (&dv)[D / 32], SPARK_LDS char* ob, int k0w,
                                        int lane, float scale) const {
    constexpr int OSTR = BwdKvPipeCfg<D>::OSTR;
    if (partial) {
      float* out = partial + (k0w >> 5 & 3) * PrefixTile<D>::WAVE + lane * 4;
#pragma unroll
      for (int q = 0; q < D / 8; ++q) {
        f32x4 a, c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] = dk[q / 4][4 * (q % 4) + e];
          c[e] = dv[q / 4][4 * (q % 4) + e];
        }
        *reinterpret_cast<f32x4*>(out + q * 256) = a;
        *reinterpret_cast<f32x4*>(out + (D / 8 + q) * 256) = c;
      }
      return;
    }
    store_transposed<T, D, OSTR>(dk, scale, ob, dK, k0w, keys, lane, (size_t)mdk.row, dh);
    store_transposed<T, D, OSTR>(dv, 1.0f, ob, dV, k0w, keys, lane, (size_t)mdv.row, dh);
  }
};

// The workgroup's part of dK and dV: `block` of first + B * Hkv * s_tiles * s_parts.
template <typename T, int D>
static __device__ __forceinline__ void prefix_dkdv(const PrefixProblem& p, const PrefixGrads<T>& gr, int p_tiles, int s_tiles,
                                                   int first, float scale, int block) {
  constexpr int BN = BwdKvPipeCfg<D>::BN;
  const int per = p.H / p.Hkv, seqs = p.B / p.G;
  const bool of_prefix = block < first;  // the longer ones first
  GroupRows<T, D> rows;
  rows.Q = static_cast<const T*>(p.Q);
  rows.dO = gr.dO;
  rows.lse2 = gr.LSE2ws;
  rows.dws = gr.Dws;
  rows.q_lens = p.q_lens;
  rows.mq = p.mq;
  rows.mdo = gr.mdo;
  rows.H = p.H;
  rows.Nq = p.Nq;
  rows.dh = p.dh;
  rows.partial = nullptr;
  int hk, tile;
  bool any = false;  // whether a row sees the tile
  bool leader = true;
  const T *K, *V;
  TensorMap mk, mv;
  if (of_prefix) {
    const int logical = xcd_contiguous(block, first);
    tile = logical % p_tiles;
    const int unit = logical / p_tiles, part = unit % gr.parts, owner = unit / gr.parts, grp = owner / p.Hkv;
    hk = owner - grp * p.Hkv;
    rows.b = grp * seqs;
    rows.b_end = rows.b + seqs;
    rows.h = rows.h0 = hk * per;
    rows.h1 = rows.h0 + per;
    rows.k0 = -1;
    leader = part == 0;
    const int stages = rows.stages(), begin = (int)((int64_t)stages * part / gr.parts);
    any = rows.start_at(begin, (int)((int64_t)stages * (part + 1) / gr.parts) - begin);
    rows.S = 0;
    rows.keys = length_of(p.prefix_lens, grp, p.P);
    rows.all = p.P;
    if (gr.parts > 1) rows.partial = gr.partial + (((size_t)part * (size_t)(p.G * p.Hkv) + owner) * (size_t)p_tiles + tile) * PrefixTile<D>::FLOATS;
    rows.dK = gr.dKp + (size_t)grp * (size_t)gr.mdkp.batch + (size_t)hk * (size_t)gr.mdkp.head;
    rows.dV = gr.dVp + (size_t)grp * (size_t)gr.mdvp.batch + (size_t)hk * (size_t)gr.mdvp.head;
    rows.mdk = gr.mdkp;
    rows.mdv = gr.mdvp;
    K = head_of<T>(p.Kp, p.mkp, grp, hk);
    V = head_of<T>(p.Vp, p.mvp, grp, hk);
    mk = p.mkp;
    mv = p.mvp;
  } else {
    // the first tiles of all suffixes first: more rows see them
    const int owners = p.B * p.Hkv, id = block - first;
    const int unit = id / owners, run = unit % gr.s_parts;
    tile = unit / gr.s_parts;
    const int owner = xcd_contiguous(id - unit * owners, owners), b = owner / p.Hkv;
    hk = owner - b * p.Hkv;
    rows.b = b;
    rows.b_end = b + 1;
    rows.h = rows.h0 = hk * per;
    rows.h1 = rows.h0 + per;
    rows.keys = rows.S = length_of(p.s_lens, b, p.S);
    rows.k0 = p.causal ? tile * BN : -1;
    const int queries = length_of(p.q_lens, b, p.Nq);
    const SuffixBlocks seen(rows.k0, p.causal ? rows.S - queries : ALL_AHEAD, queries);
    const int stages = tile * BN < rows.keys ? per * seen.count : 0, begin = run * gr.s_run;
    if (run > 0 && begin >= stages) return;
    leader = run == 0;
    if (stages > gr.s_run) rows.partial = gr.partial_s + (((size_t)run * (size_t)owners + owner) * (size_t)s_tiles + tile) * PrefixTile<D>::FLOATS;
    if (stages) any = rows.start_in(begin, seen.count, stages - begin < gr.s_run ? stages - begin : gr.s_run);
    rows.all = p.S;
    rows.dK = gr.dKs + (size_t)b * (size_t)gr.mdks.batch + (size_t)hk * (size_t)gr.mdks.head;
    rows.dV = gr.dVs + (size_t)b * (size_t)gr.mdvs.batch + (size_t)hk * (size_t)gr.mdvs.head;
    rows.mdk = gr.mdks;
    rows.mdv = gr.mdvs;
    K = head_of<T>(p.Ks, p.mks, b, hk);
    V = head_of<T>(p.Vs, p.mvs, b, hk);
    mk = p.mks;
    mv = p.mvs;
  }
  const int k0 = tile * BN, k1 = k0 + BN < rows.all ? k0 + BN : rows.all;
  const bool none = k0 >= rows.keys || !any;
  // Rows of keys that do not exist, or that no query sees: zeros, by the first of the workgroups that share the tile.  What
  // the sum reads of a part without stages: zeros too.
  const int from = none && !rows.partial ? k0 : rows.keys > k0 ? rows.keys : k0;
  if (from < k1 && leader) {
    zero_rows(rows.dK, rows.mdk, from, k1, p.dh);
    zero_rows(rows.dV, rows.mdv, from, k1, p.dh);
  }
  if (none && rows.partial) {
    for (int i = threadIdx.x; i < PrefixTile<D>::FLOATS / 4; i += 256)
      reinterpret_cast<f32x4*>(rows.partial)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (none) return;
  const TensorMap none_map{0, 0, 0};
  if (of_prefix)
    bwd_dkdv_pipe<T, D, false, false, IN_ORDER, false>(nullptr, K, V, nullptr, nullptr, nullptr, nullptr, nullptr, p.mq, mk, mv,
                                                       gr.mdo, none_map, none_map, 1, p.Nq, rows.keys, p.dh, p_tiles, 0, scale,
                                                       Dropout{}, 0, tile, rows);
  else
    bwd_dkdv_pipe<T, D, true, false, IN_ORDER, false>(nullptr, K, V, nullptr, nullptr, nullptr, nullptr, nullptr, p.mq, mk, mv,
                                                      gr.mdo, none_map, none_map, 1, p.Nq, rows.keys, p.dh, s_tiles, 0, scale,
                                                      Dropout{}, 0, tile, rows);
}

template <typename T, int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void mha_prefix_dkdv_kernel(PrefixProblem p, PrefixGrads<T> gr,
                                                                               int p_tiles, int s_tiles, int first,
                                                                               float scale) {
  prefix_dkdv<T, D>(p, gr, p_tiles, s_tiles, first, scale, blockIdx.x);
}

// Both in one grid where one of them leaves CUs idle: the workgroups of the prefix's keys, those of dQ, those of the suffixes'.
// D and LSE * log2(e) are formed by a kernel of their own first.
template <typename T, int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void mha_prefix_bwd_kernel(PrefixProblem p, PrefixGrads<T> gr, int p_tiles,
                                                                              int s_tiles, int first, int nqt, float scale) {
  const int dq_items = p.B * p.Hkv * nqt * gr.q_parts, block = blockIdx.x;
  if (block >= first && block < first + dq_items)
    prefix_dq<T, D, true>(p, nullptr, gr, nqt, scale, xcd_contiguous(block - first, dq_items));
  else
    prefix_dkdv<T, D>(p, gr, p_tiles, s_tiles, first, scale, block < first ? block : block - dq_items);
}

// -D and LSE * log2(e) of every row: W / 8 lanes to a row.  A row without keys gets inf, so that its P is 0; rows not in use are
// never read.
template <typename T, int W>
__global__ __launch_bounds__(256) void mha_prefix_stats_kernel(PrefixProblem p, const T* __restrict__ O, PrefixGrads<T> gr) {
  using v8 = typename Frag<T>::v8;
  constexpr int LPR = W / 8;
  const size_t rows = (size_t)p.B * p.H * (size_t)p.Nq, row = (size_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const size_t r = row < rows ? row : rows - 1;
  const int bh = (int)(r / (size_t)p.Nq), i = (int)(r - (size_t)bh * p.Nq), b = bh / p.H, h = bh - b * p.H;
  const int col = (threadIdx.x % LPR) * 8;
  const bool used = row < rows && i < length_of(p.q_lens, b, p.Nq);
  const v8 o = load_row_chunk<v8>(head_of<T>(O, p.mo, b, h) + (size_t)i * (size_t)p.mo.row, col, p.dh);
  const v8 g = load_row_chunk<v8>(head_of<T>(gr.dO, gr.mdo, b, h) + (size_t)i * (size_t)gr.mdo.row, col, p.dh);
  float acc = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc = __builtin_fmaf((float)o[e], (float)g[e], acc);
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) acc += __shfl_xor(acc, m, LPR);
  if (used && col == 0) {
    const float lse = gr.LSE[r];
    gr.Dws[r] = -acc;
    gr.LSE2ws[r] = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
  }
}

// Sum of the parts of 32 rows of a tile, in their order, times `mul_first` in the first `first` eights of columns; rounded into
// `rows`.  1024 threads; four parts are requested together.
template <typename T, int EIGHTS>
static __device__ __forceinline__ void sum_parts(const float* x, size_t step, int parts, int first, float mul_first,
                                                 T (&rows)[32][8 * EIGHTS + 8]) {
  using v4 = typename Frag<T>::v4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x += lane * 4;
#pragma unroll
  for (int q = wave; q < EIGHTS; q += 16) {
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < parts; i += 4) {
      f32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const f32x4*>(x + (i + u < parts ? i + u : i) * step + q * 256);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i + u < parts) a += v[u];
      }
    }
    const float mul = q < first ? mul_first : 1.0f;
    v4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (T)(a[e] * mul);
    *reinterpret_cast<v4*>(&rows[lane & 31][8 * q + 4 * (lane >> 5)]) = r;
  }
  __syncthreads();
}

// Gradients of the tiles that several workgroups share: a workgroup per 32 rows, first of the prefixes' keys (p_blocks
// workgroups), then of the suffixes' (s_blocks), then of the queries.
template <typename T, int D>
__global__ __launch_bounds__(1024) void mha_prefix_sum_kernel(PrefixProblem p, PrefixGrads<T> gr, int p_blocks, int s_blocks,
                                                              int p_tiles, int s_tiles, int nqt, float scale) {
  using Tile = PrefixTile<D>;
  const int block = blockIdx.x;
  if (block >= p_blocks + s_blocks) {
    __shared__ __align__(16) T rows[32][D + 8];
    const int id = block - p_blocks - s_blocks, quarter = id & 3, at = id >> 2, owner = at / nqt, tile = at - owner * nqt,
              b = owner / p.Hkv, hk = owner - b * p.Hkv, per = p.H / p.Hkv, row0 = tile * 128 + quarter * 32;
    // what no workgroup took on is zero already
    const int q = length_of(p.q_lens, b, p.Nq), S = length_of(p.s_lens, b, p.S), P = length_of(p.prefix_lens, b / (p.B / p.G), p.P);
    const int all = p.Nq * per, end = tile * 128 + 128 < all ? tile * 128 + 128 : all;
    if (tile * 128 >= q * per || (P == 0 && (S == 0 || (end - 1) / per + (p.causal ? S - q : ALL_AHEAD) < 0))) return;
    const size_t step = (size_t)p.B * (size_t)p.Hkv * (size_t)nqt * Tile::Q_FLOATS;
    sum_parts<T, D / 8>(gr.partial_q + (size_t)at * Tile::Q_FLOATS + quarter * Tile::Q_WAVE, step, gr.q_parts, D / 8, scale, rows);
    T* const dQ = gr.dQ + (size_t)b * (size_t)gr.mdq.batch + (size_t)(hk * per) * (size_t)gr.mdq.head;
    for (int i = threadIdx.x; i < 32 * (D / 8); i += 1024) {
      const int r = row0 + i / (D / 8), col = i % (D / 8) * 8, query = r / per;
      if (r >= all || col >= p.dh) continue;
      *reinterpret_cast<u32x4*>(dQ + (size_t)query * (size_t)gr.mdq.row + (size_t)(r - query * per) * (size_t)gr.mdq.head + col) =
          *reinterpret_cast<const u32x4*>(&rows[r - row0][col]);
    }
    return;
  }
  __shared__ __align__(16) T rows[32][2 * D + 8];
  const bool of_prefix = block < p_blocks;
  const int id = of_prefix ? block : block - p_blocks, quarter = id & 3, at = id >> 2;
  const int tiles = of_prefix ? p_tiles : s_tiles, owner = at / tiles, tile = at - owner * tiles, outer = owner / p.Hkv,
            hk = owner - outer * p.Hkv, key0 = tile * 128 + quarter * 32;
  int parts = gr.parts, keys;
  if (of_prefix) {
    keys = length_of(p.prefix_lens, outer, p.P);
  } else {
    keys = length_of(p.s_lens, outer, p.S);
    const int queries = length_of(p.q_lens, outer, p.Nq);
    const SuffixBlocks seen(p.causal ? tile * 128 : -1, p.causal ? keys - queries : ALL_AHEAD, queries);
    const int stages = p.H / p.Hkv * seen.count;
    if (stages <= gr.s_run) return;  // one workgroup's, in place already
    parts = (stages + gr.s_run - 1) / gr.s_run;
  }
  if (key0 >= keys) return;  // zeros already
  const size_t step = (size_t)(of_prefix ? p.G : p.B) * (size_t)p.Hkv * (size_t)tiles * Tile::FLOATS;
  sum_parts<T, Tile::EIGHTS>((of_prefix ? gr.partial : gr.partial_s) + (size_t)at * Tile::FLOATS + quarter * Tile::WAVE, step, parts,
                             D / 8, scale, rows);
  T* const dK = of_prefix ? gr.dKp : gr.dKs;
  T* const dV = of_prefix ? gr.dVp : gr.dVs;
  const TensorMap &mk = of_prefix ? gr.mdkp : gr.mdks, &mv = of_prefix ? gr.mdvp : gr.mdvs;
  for (int i = threadIdx.x; i < 32 * (2 * D / 8); i += 1024) {
    const int row = i / (2 * D / 8), c = i % (2 * D / 8), col = c % (D / 8) * 8, key = key0 + row;
    if (key >= keys || col >= p.dh) continue;
    const TensorMap& m = c < D / 8 ? mk : mv;
    T* const out = (c < D / 8 ? dK : dV) + (size_t)outer * (size_t)m.batch + (size_t)hk * (size_t)m.head + (size_t)key * (size_t)m.row;
    *reinterpret_cast<u32x4*>(out + col) = *reinterpret_cast<const u32x4*>(&rows[row][8 * c]);
  }
}

}  // namespace spark
