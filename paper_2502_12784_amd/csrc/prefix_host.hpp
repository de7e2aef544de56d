// Host side of spark_mha_prefix_*: argument checks, launch shapes, dispatch.
#pragma once
#include "host_util.hpp"
#include "prefix_kernels.hpp"
#include "prefix_parts.hpp"

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
  // packed rows of a sequence (query, head) are counted in 31 bits, and so are a tile's worth more
  if ((int64_t)Nq * (H / Hkv) >= (int64_t)1 << 30) return SPARK_ERR_SHAPE;
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
  const int nqt = (p.Nq * (p.H / p.Hkv) + C::BM - 1) / C::BM;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.B * p.Hkv * nqt)), dim3(64 * NW), C::SMEM, st, p, static_cast<T*>(O), LSE, nqt,
                     scale * 1.4426950408889634f);
  return launch_ok("forward kernel (prefix)") ? SPARK_OK : SPARK_ERR_LAUNCH;
}

// Workgroups of 8 waves (256 rows, one per CU) instead of 4: the rule of wide_workgroups in spark_mha.hip, for the same loop;
// not where the last of few tiles would stay half empty (us, 64 sequences x 32 heads over 8 x 16 queries behind 2048, one
// half tile each: 118 in wide ones, 71).
bool prefix_wide(const PrefixProblem& p) {
  const int64_t rows = (int64_t)p.Nq * (p.H / p.Hkv), owners = (int64_t)p.B * p.Hkv;
  const int64_t wide = owners * ((rows + 255) / 256), narrow = owners * ((rows + 127) / 128);
  return (int64_t)p.P + p.S >= 2048 && 7 * wide <= 4 * narrow && (wide >= 512 || narrow >= 896 || (wide <= 256 && narrow > 256));
}

// Whether rows are packed across sequences and the keys go to several workgroups in runs (prefix_parts.hpp), or every tile of a
// sequence's rows walks all its keys by itself: where those tiles fill the chip and are well filled themselves.  Forward, us,
// d = 128 but where said, packed / by themselves:
//   rows of a tile in use, half: 32 x 16 x 64 behind 1024 42.5 / 36.7, d = 64 28.4 / 24.9; 64 x 32 over 8 x 16 behind 2048 62.6 / 70.6;
//   a third: 64 x 16 x 48 behind 2048 82.8 / 125, 32 x 16 x 40 behind 1024 32.4 / 35.4; a quarter: 64 x 16 x 32 behind 2048 57 / 119;
//   three quarters: 16 x 16 x 96 behind 1024 36.2 / 27.0, 16 x 64 over 16 x 24 behind 2048 47.5 / 40.6
//   few tiles (n): 2 x 16 x 256 behind 4096 (64) 35 / 73, 4 x 16 x 256 (128) 55 / 74, 8 x 16 x 160 behind 2048 (256) 46.0 / 43.6
bool prefix_packed(const PrefixProblem& p) {
  const int64_t rows = (int64_t)p.Nq * (p.H / p.Hkv), tiles = (rows + 127) / 128;
  if (p.B * (int64_t)p.Hkv * tiles < 256) return true;
  const int64_t filled = 100 * rows / (128 * tiles);  // percent of the tiles' rows
  return filled < (p.P <= 1280 ? 48 : 60);
}

// Whether 32 packed rows of a sequence go to a workgroup with all their keys (mha_prefix_short_kernel): a chain of keys / 256 rounds
// (at 64 columns / 512; of four waves instead of eight, half of that) and no merge, against runs of keys and a merge
// (prefix_packed).  Returns its waves: eight up to one workgroup per CU, four, two workgroups to a CU, for more of them or few
// keys; 0: not so.  Forward, us, in runs / so (n workgroups, keys):
//   d = 128:  56: 1088 13.6 / 12.9, 2112 16.9 / 18.0    64: 2112 19.0 / 17.9, 4160 24.4 / 28.1   128: 1088 16.6 / 14.6, 2112 20.1 / 20.3
//             256: 1088 16.1 / 14.1, 2112 27.8 / 20.4, or 23.0 / 21.5 at 40 rows a sequence, then 4160 30.3 / 35.0
//             512: 1274 30.7 / 23.8, 2298 37.3 / 36.8, 4346 53.5 / 60.6              768: 576 29.5 / 24.7, 1088 33.6 / 33.9
//   d = 64:   56: 1088 10.6 / 9.6, 2112 12.0 / 12.2     64: 2112 13.0 / 12.5, 4160 18.8 / 17.9   128: 2112 14.4 / 13.7, 4160 18.3 / 19.5
//             256: 2112 16.8 / 13.4, 4160 25.5 / 19.7, or 21.4 / 21.9 at 40 rows
//             512: 1274 23.5 / 15.5, 2298 26.0 / 22.2, 4346 34.6 / 34.6              768: 1088 24.9 / 22.7, 2112 33.9 / 33.8
//   against tiles of 128 rows by themselves (1024 workgroups so) 576 keys d = 128 17.5 / 28.0, d = 64 13.1 / 19.7;
//   four waves / eight: 64 workgroups d = 64 264 keys 7.2 / 7.5, 564 8.4 / 8.3, 2112 15.3 / 12.5, d = 128 264 9.0 / 9.3, 2112 23.9 / 17.9.
// Where a sequence's rows fill a part of one workgroup only, packing reads the prefix once for several sequences, and the limit falls
// with the rows (sequences x heads x queries, keys):
//   d = 128:  32 x 16 x 1 320 13.9 / 11.8, 448 14.0 / 13.2, 704 14.4 / 16.1; 32 x 16 over 8 x 1 564 11.3 / 10.7, 1088 11.9 / 13.8;
//             8 x 16 x 16 1088 15.5 / 13.5, 2112 18.7 / 18.8; 4 x 32 over 8 x 1 328 9.4 / 8.6, 712 9.8 / 11.8
//   d = 64:   2 x 4 x 1 564 8.1 / 8.0, 1088 8.6 / 9.4; 32 x 16 over 8 x 1 564 8.6 / 8.5, 1088 9.3 / 10.0; 8 x 16 x 16 2112 13.3 / 12.5
int prefix_short(const PrefixProblem& p) {
  const int64_t rows = (int64_t)p.Nq * (p.H / p.Hkv), tiles = (rows + 31) / 32, groups = p.B * (int64_t)p.Hkv * tiles;
  const int64_t n = (int64_t)p.P + p.S;
  const bool narrow = p.dh <= 64;
  const int64_t few = narrow ? 640 : 512;
  int64_t most = few;  // keys
  if (groups <= 256) {
    const int64_t line = narrow ? 384 + 32 * groups : 256 + 24 * groups, top = narrow ? 4096 : 2400;
    most = line < top ? line : top;
  } else if (groups <= 512) {
    most = narrow ? 3200 : 2048;
  } else if (groups <= 768 && prefix_packed(p)) {
    most = narrow ? 2048 : 1024;
  } else if (tiles > 1) {
    return 0;
  }
  if (most < few) most = few;
  if (tiles == 1) most = few + (most - few) * rows / 32;
  return n > most ? 0 : groups <= 256 && n > 512 ? 8 : 4;
}

// The runs of keys.  Two workgroups fit a CU, 512 in all.  Up to 96 packed rows the prefix is read by tiles of 32 rows, beyond that
// multiplied in tiles of 128 (us, 80 rows, 4001 keys, d = 64: 16.4, in one tile of 128 18.4).  Its runs fill half of the chip's
// places; a prefix that is only read leaves them to the suffixes where these fill them anyway (us, 32 sequences x 16 heads, 4096 keys,
// 64 / 96 / 128 / 192 / 256 workgroups 23.1 / 23.0 / 23.8 / 25.6 / 25.9; 96 suffixes, 4001 keys 23.4 / 23.8 / 23.5 / 16.7 / 16.1).
// A prefix that is multiplied leaves some to suffixes with as much work, tiles times keys, as its own (32 heads over 8, us, the
// ratio of the work in front, d = 64 and 128, 128 / 192 / 224 / 256 workgroups; more of them are slower everywhere):
//   0.1   32 x 5 behind 16384 + 300    65.7 / 52.1 / 45.2 / 41.8     93.6 / 76.1 / 68.8 / 67.3
//   0.6   48 x 1 behind 8192 + 200     20.8 / 18.3 / 19.8 / 21.7     28.5 / 26.3 / 27.3 / 28.8
//   1     128 x 1 behind 8192 + 256    33.3 / 31.1 / 32.0 / 33.5     53.2 / 49.2 / 50.4 / 53.0
//   1     64 x 1 behind 16384 + 512    35.2 / 31.2 / 29.2 / 31.6     56.6 / 50.2 / 48.6 / 49.5
//   4     128 x 1 behind 8192 + 1024   54.0 / 56.6 / 56.9 / 57.5     94.5 / 98.2 / 98.0 / 101.7
PrefixParts prefix_runs(const PrefixProblem& p) {
  PrefixParts s{};
  const int64_t per = p.H / p.Hkv, rows = (int64_t)(p.B / p.G) * p.Nq * per;
  const int bn = p.dh <= 64 ? 64 : 32;
  s.wide = rows > 96;
  s.p_tiles = p.P ? (int)((rows + (s.wide ? 127 : 31)) / (s.wide ? 128 : 32)) : 0;
  s.s_tiles = p.S ? (int)((p.Nq * per + 31) / 32) : 0;
  const int64_t n1 = (int64_t)p.G * p.Hkv * s.p_tiles, n2 = (int64_t)p.B * p.Hkv * s.s_tiles;
  // 64 runs at most (16 instead, of one sequence's suffix alone, d = 128, 8 heads over 1, 65536 keys 32.7 us, so 16.3; 32 over 8,
  // 131072 keys 107.6, 97.5)
  auto runs = [](int64_t places, int64_t items, int64_t units) {
    int64_t n = items ? places / items : 0;
    if (n > units) n = units;
    if (n > 64) n = 64;
    return (int)(n < 1 ? 1 : n);
  };
  const int64_t p_work = n1 * p.P, s_work = n2 * p.S;
  const int64_t beside = 5 * s_work < 2 * p_work ? 256 : s_work < 2 * p_work ? 208 : 128;
  const int64_t places = s.wide ? beside : n2 <= 256 ? 256 : n2 >= 416 ? 96 : 512 - n2;
  // at least four tiles of the wide loop to a run, or two rounds of the four key streams
  s.p_parts = p.P ? runs(places, n1, s.wide ? (p.P + 255) / 256 : (p.P + 8 * bn - 1) / (8 * bn)) : 0;
  s.s_parts = p.S ? runs(256, n2, (p.S + 8 * bn - 1) / (8 * bn)) : 0;
  s.p_items = (int)(n1 * s.p_parts);
  return s;
}
size_t prefix_fwd_workspace(const PrefixProblem& p) {
  if (prefix_short(p) || !prefix_packed(p)) return 0;
  const PrefixParts s = prefix_runs(p);
  return (size_t)p.B * p.H * p.Nq * (size_t)(s.p_parts + s.s_parts) * ((p.dh <= 64 ? 64 : 128) + 4) * sizeof(float);
}

template <typename T, int D>
int launch_prefix_parts(const PrefixProblem& p, void* O, float* LSE, void* workspace, float scale, hipStream_t st) {
  constexpr int W = lds_row<D>, SMEM = FwdCfg<D>::SMEM > FwdSplitCfg<W, 4>::SMEM ? FwdCfg<D>::SMEM : FwdSplitCfg<W, 4>::SMEM;
  auto kernel = mha_prefix_parts_kernel<T, D>;
  static std::atomic<uint64_t> ready{0};
  const int attr = ensure_smem(kernel, SMEM, ready);
  if (attr != SPARK_OK) return attr;
  PrefixParts s = prefix_runs(p);
  s.partial = static_cast<float*>(workspace);
  const int grid = s.p_items + p.B * p.Hkv * s.s_tiles * s.s_parts;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), SMEM, st, p, s, scale * 1.4426950408889634f);
  if (!launch_ok("forward kernel (prefix, in runs)")) return SPARK_ERR_LAUNCH;
  // four parts are requested by a lane together: as many lanes side by side to a row as that leaves
  const int parts = s.p_parts + s.s_parts;
  const int64_t rows = (int64_t)p.B * p.H * p.Nq;
  constexpr int MOST = 256 / (W / 4);
  auto merge = parts <= 4    ? mha_prefix_merge_kernel<T, W, 1>
               : parts <= 8  ? mha_prefix_merge_kernel<T, W, 2>
               : parts <= 16 ? mha_prefix_merge_kernel<T, W, 4>
                             : mha_prefix_merge_kernel<T, W, MOST>;
  const int side = parts <= 4 ? 1 : parts <= 8 ? 2 : parts <= 16 ? 4 : MOST, each = MOST / side;
  hipLaunchKernelGGL(merge, dim3((unsigned)((rows + each - 1) / each)), dim3(256), 0, st, p, s.partial, parts,
                     static_cast<T*>(O), LSE);
  return launch_ok("forward merge kernel (prefix)") ? SPARK_OK : SPARK_ERR_LAUNCH;
}

template <typename T, int W, int NW>
int launch_prefix_short(const PrefixProblem& p, void* O, float* LSE, float scale, hipStream_t st) {
  using C = FwdSplitCfg<W, NW>;
  auto kernel = mha_prefix_short_kernel<T, W, NW>;
  static std::atomic<uint64_t> ready{0};
  const int attr = ensure_smem(kernel, C::SMEM, ready);
  if (attr != SPARK_OK) return attr;
  const int nqt = (p.Nq * (p.H / p.Hkv) + 31) / 32;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.B * p.Hkv * nqt)), dim3(64 * NW), C::SMEM, st, p, static_cast<T*>(O), LSE, nqt,
                     scale * 1.4426950408889634f);
  return launch_ok("forward kernel (prefix, few keys)") ? SPARK_OK : SPARK_ERR_LAUNCH;
}

template <typename T>
int dispatch_prefix_fwd(const PrefixProblem& p, void* O, float* LSE, void* workspace, float scale, hipStream_t st) {
  const int waves = prefix_short(p);
  if (waves == 8)
    return p.dh <= 64 ? launch_prefix_short<T, 64, 8>(p, O, LSE, scale, st) : launch_prefix_short<T, 128, 8>(p, O, LSE, scale, st);
  if (waves)
    return p.dh <= 64 ? launch_prefix_short<T, 64, 4>(p, O, LSE, scale, st) : launch_prefix_short<T, 128, 4>(p, O, LSE, scale, st);
  if (workspace && prefix_packed(p)) {
    if (p.dh <= 64) return launch_prefix_parts<T, 64>(p, O, LSE, workspace, scale, st);
    if (p.dh <= 96) return launch_prefix_parts<T, 96>(p, O, LSE, workspace, scale, st);
    return launch_prefix_parts<T, 128>(p, O, LSE, workspace, scale, st);
  }
  if (p.dh <= 64) return launch_prefix_fwd<T, 64, 4, false>(p, O, LSE, scale, st);
  const bool wide = prefix_wide(p);
  if (p.dh <= 96) return wide ? launch_prefix_fwd<T, 96, 8, true>(p, O, LSE, scale, st) : launch_prefix_fwd<T, 96, 4, false>(p, O, LSE, scale, st);
  return wide ? launch_prefix_fwd<T, 128, 8, true>(p, O, LSE, scale, st) : launch_prefix_fwd<T, 128, 4, false>(p, O, LSE, scale, st);
}

// How many workgroups share the rows of a key tile in the dK/dV kernel, by an estimate of its time.  Counted in stages (64 rows
// of a head against 128 keys, some 2 us): a workgroup costs three more, the parts of dKp and dVp are written and read once,
// and the end of the grid waits for half a short item.  A suffix tile is cut into runs of half a prefix tile's stages, at least
// four.  (us, step of 6 sequences x 6 heads over 2 x 333 behind 700, d = 80, 1 / 3 / 5 / 6 parts with whole suffix tiles - / 77 / 89 / 90;
// 16 sequences x 16 over 4 x 512 behind 1024, 2 / 3 / 4 / 6 parts 399 / 386 / 392 / 385.)
struct PrefixShares {
  int parts, s_parts, s_run;
};
PrefixShares prefix_shares(const PrefixProblem& p) {
  const double slots = 256 * (p.dh <= 64 ? 2 : 1), columns = p.dh <= 64 ? 64 : p.dh <= 96 ? 96 : 128;
  const int64_t per = p.H / p.Hkv, blocks = (p.Nq + 63) / 64;
  const int64_t n1 = (int64_t)p.G * p.Hkv * ((p.P + 127) / 128), n2 = (int64_t)p.B * p.Hkv * ((p.S + 127) / 128);
  const int64_t w1 = p.B / p.G * per * blocks, w2 = per * blocks;
  auto run_of = [&](int64_t parts) {
    int64_t run = p.P ? w1 / parts / 2 : (n2 * w2 + 511) / 512;
    if (run < 4) run = 4;
    if (run < (w2 + 15) / 16) run = (w2 + 15) / 16;  // sixteen runs at most
    return run < w2 ? run : w2;
  };
  int64_t best = 1;
  double least = 0;
  for (int64_t parts = 1; parts <= 32 && parts <= w1 && p.P; ++parts) {
    const double run = (double)run_of(parts), item = (double)w1 / parts + 3, runs = (double)((w2 + (int64_t)run - 1) / (int64_t)run);
    const double s_item = run + 3, s_work = (p.causal ? 0.5 : 1.0) * w2 + 3 * runs;
    const double work = (n1 * parts * item + n2 * s_work) / slots, longest = item > s_item ? item : s_item;
    double time = work + (item < s_item ? item : s_item) / 2;
    if (n1 * parts + n2 * runs <= slots || time < longest) time = longest;
    if (parts > 1) time += parts * n1 * 128.0 * columns * 16 / 8e6;
    if (parts == 1 || time < least) {
      best = parts;
      least = time;
    }
  }
  if (n1 * best >= (int64_t)1 << 30) best = 1;
  int64_t run = run_of(best);
  if (n2 * ((w2 + run - 1) / run) >= (int64_t)1 << 30) run = w2;
  return PrefixShares{(int)best, p.S ? (int)((w2 + run - 1) / run) : 1, (int)run};
}
size_t prefix_stats_bytes(const PrefixProblem& p) { return ((size_t)p.B * p.H * p.Nq * 8 + 255) & ~(size_t)255; }
// Floats of the parts of all prefix tiles, and of all suffix tiles (PrefixTile).
size_t part_floats(const PrefixProblem& p, int parts, int outer, int n) {
  const size_t columns = p.dh <= 64 ? 64 : p.dh <= 96 ? 96 : 128;
  return parts > 1 ? (size_t)parts * outer * p.Hkv * ((n + 127) / 128) * 128 * 2 * columns : 0;
}
size_t prefix_part_floats(const PrefixProblem& p, const PrefixShares& x) { return part_floats(p, x.parts, p.G, p.P); }
size_t suffix_part_floats(const PrefixProblem& p, const PrefixShares& x) { return part_floats(p, x.s_parts, p.B, p.S); }
// Workgroups that share the keys of a tile of rows in dQ: as many as give every place (two to a CU) one, with eight tiles of
// keys to each at least, sixteen at most.  (Steps, us, one -> so: 1 head x 192 queries behind 8192 keys, d = 128, 223 -> 44;
// 2 sequences x 32 heads over 8 x 128 behind 8192, d = 128, 363 -> 246; 5 x 1 x 23 behind 4672, d = 64, 76 -> 33.)
int64_t dq_tiles(const PrefixProblem& p) { return (int64_t)p.B * p.Hkv * (((int64_t)p.Nq * (p.H / p.Hkv) + 127) / 128); }
int query_parts(const PrefixProblem& p) {
  const int64_t tiles = ((int64_t)p.P + p.S + 63) / 64 * (p.dh > 96 ? 2 : 1);
  int64_t parts = 512 / dq_tiles(p);
  if (parts > tiles / 8) parts = tiles / 8;
  return parts > 16 ? 16 : parts < 1 ? 1 : (int)parts;
}
size_t query_part_floats(const PrefixProblem& p) {
  const int parts = query_parts(p);
  return parts > 1 ? (size_t)parts * (size_t)dq_tiles(p) * 128 * (p.dh <= 64 ? 64 : p.dh <= 96 ? 96 : 128) : 0;
}
size_t prefix_bwd_workspace(const PrefixProblem& p) {
  const PrefixShares x = prefix_shares(p);
  return prefix_stats_bytes(p) + sizeof(float) * (prefix_part_floats(p, x) + suffix_part_floats(p, x) + query_part_floats(p));
}

// Whether dQ and dK/dV run in one grid: where dQ's tiles alone leave CUs idle.  In one grid dQ, which has two workgroups to a
// CU by itself, is held to one at more than 64 columns.  Steps, us, a grid for each -> one grid (n tiles of dQ):
//   d = 64:   2 sequences x 8 heads over 2 x 128 queries behind 256 (16) 34.5 -> 27.5   8 x 8 x 512 behind 1024 (256) 88.2 -> 86.4
//             4 x 8 x 512 behind 4096 (128) 152.8 -> 138.4                               16 x 8 x 512 behind 1024 (512) 137.9 -> 132.6
//   d <= 96:  6 x 6 over 2 x 333 behind 700 (96) 81.5 -> 68.1                            8 x 12 x 384 behind 512 (288) 106.5 -> 100.5
//   d = 128:  4 x 16 over 4 x 256 behind 512 (128) 88.4 -> 83.9                          8 x 16 x 256 behind 1024 (256) 131.0 -> 136.2
//             8 x 16 over 4 x 512 behind 2048 (512) 311.7 -> 354.9
bool prefix_merged(const PrefixProblem& p) {
  return dq_tiles(p) <= (p.dh <= 64 ? 512 : p.dh <= 96 ? 288 : 192);
}

template <typename T, int D>
int launch_prefix_bwd(const PrefixProblem& p, const void* O, PrefixGrads<T> gr, float scale, bool merged, hipStream_t st) {
  using Q = BwdQCfg<D, true, false>;
  using C = BwdKvPipeCfg<D>;
  const int nqt = (p.Nq * (p.H / p.Hkv) + Q::BM - 1) / Q::BM, dq_items = p.B * p.Hkv * nqt * gr.q_parts;
  const int p_tiles = (p.P + C::BN - 1) / C::BN, s_tiles = (p.S + C::BN - 1) / C::BN;
  const int first = p.G * p.Hkv * gr.parts * p_tiles, grid = first + p.B * p.Hkv * s_tiles * gr.s_parts;
  if (merged) {
    constexpr int W = lds_row<D>, RPB = 256 / (W / 8), SMEM = C::SMEM > Q::SMEM ? C::SMEM : Q::SMEM;
    const int64_t rows = (int64_t)p.B * p.H * p.Nq;
    hipLaunchKernelGGL((mha_prefix_stats_kernel<T, W>), dim3((unsigned)((rows + RPB - 1) / RPB)), dim3(256), 0, st, p,
                       static_cast<const T*>(O), gr);
    if (!launch_ok("backward statistics kernel (prefix)")) return SPARK_ERR_LAUNCH;
    auto kernel = mha_prefix_bwd_kernel<T, D>;
    static std::atomic<uint64_t> ready{0};
    const int attr = ensure_smem(kernel, SMEM, ready);
    if (attr != SPARK_OK) return attr;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(grid + dq_items)), dim3(256), SMEM, st, p, gr, p_tiles, s_tiles, first, nqt, scale);
    if (!launch_ok("backward kernel (prefix, both sides)")) return SPARK_ERR_LAUNCH;
  } else {
    {
      auto kernel = mha_prefix_dq_kernel<T, D>;
      static std::atomic<uint64_t> ready{0};
      const int attr = ensure_smem(kernel, Q::SMEM, ready);
      if (attr != SPARK_OK) return attr;
      hipLaunchKernelGGL(kernel, dim3((unsigned)dq_items), dim3(256), Q::SMEM, st, p, static_cast<const T*>(O), gr, nqt, scale);
      if (!launch_ok("dQ kernel (prefix)")) return SPARK_ERR_LAUNCH;
    }
    auto kernel = mha_prefix_dkdv_kernel<T, D>;
    static std::atomic<uint64_t> ready{0};
    const int attr = ensure_smem(kernel, C::SMEM, ready);
    if (attr != SPARK_OK) return attr;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), C::SMEM, st, p, gr, p_tiles, s_tiles, first, scale);
    if (!launch_ok("dK/dV kernel (prefix)")) return SPARK_ERR_LAUNCH;
  }
  if (gr.parts == 1 && gr.s_parts == 1 && gr.q_parts == 1) return SPARK_OK;
  const int p_blocks = gr.parts > 1 ? p.G * p.Hkv * p_tiles * 4 : 0, s_blocks = gr.s_parts > 1 ? p.B * p.Hkv * s_tiles * 4 : 0;
  const int q_blocks = gr.q_parts > 1 ? p.B * p.Hkv * nqt * 4 : 0;
  hipLaunchKernelGGL((mha_prefix_sum_kernel<T, D>), dim3((unsigned)(p_blocks + s_blocks + q_blocks)), dim3(1024), 0, st, p, gr,
                     p_blocks, s_blocks, p_tiles, s_tiles, nqt, scale);
  return launch_ok("sum of the parts (prefix)") ? SPARK_OK : SPARK_ERR_LAUNCH;
}

struct PrefixGradArgs {
  const void* dO;
  void *dQ, *dKp, *dVp, *dKs, *dVs;
  TensorMap mdo, mdq, mdkp, mdvp, mdks, mdvs;
  const float* LSE;
  void* workspace;
};

template <typename T>
int dispatch_prefix_bwd(const PrefixProblem& p, const void* O, const PrefixGradArgs& a, float scale, hipStream_t st) {
  PrefixGrads<T> gr;
  gr.dO = static_cast<const T*>(a.dO);
  gr.dQ = static_cast<T*>(a.dQ);
  gr.dKp = static_cast<T*>(a.dKp);
  gr.dVp = static_cast<T*>(a.dVp);
  gr.dKs = static_cast<T*>(a.dKs);
  gr.dVs = static_cast<T*>(a.dVs);
  gr.mdo = a.mdo; gr.mdq = a.mdq; gr.mdkp = a.mdkp; gr.mdvp = a.mdvp; gr.mdks = a.mdks; gr.mdvs = a.mdvs;
  gr.LSE = a.LSE;
  gr.Dws = static_cast<float*>(a.workspace);
  gr.LSE2ws = gr.Dws + (size_t)p.B * p.H * p.Nq;
  gr.partial = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + prefix_stats_bytes(p));
  const PrefixShares x = prefix_shares(p);
  gr.parts = x.parts;
  gr.s_parts = x.s_parts;
  gr.s_run = x.s_run;
  gr.partial_s = gr.partial + prefix_part_floats(p, x);
  gr.q_parts = query_parts(p);
  gr.partial_q = gr.partial_s + suffix_part_floats(p, x);
  const bool merged = prefix_merged(p);
  if (p.dh <= 64) return launch_prefix_bwd<T, 64>(p, O, gr, scale, merged, st);
  if (p.dh <= 96) return launch_prefix_bwd<T, 96>(p, O, gr, scale, merged, st);
  return launch_prefix_bwd<T, 128>(p, O, gr, scale, merged, st);
}

}  // namespace

extern "C" {

size_t spark_mha_prefix_bwd_workspace_bytes(int G, int B, int H, int Hkv, int Nq, int P, int S, int d, int causal,
                                            spark_dtype_t dtype) {
  PrefixProblem p{};
  if (make_prefix(&p, G, B, H, Hkv, Nq, P, S, d, 1.0f, causal, (int)dtype) != SPARK_OK) return 0;
  return prefix_bwd_workspace(p);
}

int spark_mha_prefix_bwd(const void* Q, const void* Kp, const void* Vp, const void* Ks, const void* Vs, const void* O,
                         const float* LSE, const void* dO, void* dQ, void* dKp, void* dVp, void* dKs, void* dVs,
                         const spark_strides_t* sQ, const spark_strides_t* sKp, const spark_strides_t* sVp,
                         const spark_strides_t* sKs, const spark_strides_t* sVs, const spark_strides_t* sO,
                         const spark_strides_t* sdO, const spark_strides_t* sdQ, const spark_strides_t* sdKp,
                         const spark_strides_t* sdVp, const spark_strides_t* sdKs, const spark_strides_t* sdVs,
                         const int* prefix_lens, const int* q_lens, const int* s_lens, void* workspace,
                         size_t workspace_bytes, int G, int B, int H, int Hkv, int Nq, int P, int S, int d, float scale,
                         int causal, spark_dtype_t dtype, void* stream) {
  if (!Q || !O || !LSE || !dO || !dQ || !workspace) return SPARK_ERR_NULL;
  PrefixProblem p{};
  PrefixGradArgs a{};
  int rc = make_prefix(&p, G, B, H, Hkv, Nq, P, S, d, scale, causal, (int)dtype);
  if (rc != SPARK_OK) return rc;
  if ((rc = check_part(Q, sQ, B, H, Nq, d, false, &p.mq)) != SPARK_OK) return rc;
  if ((rc = check_part(Kp, sKp, G, Hkv, P, d, false, &p.mkp)) != SPARK_OK) return rc;
  if ((rc = check_part(Vp, sVp, G, Hkv, P, d, false, &p.mvp)) != SPARK_OK) return rc;
  if ((rc = check_part(Ks, sKs, B, Hkv, S, d, false, &p.mks)) != SPARK_OK) return rc;
  if ((rc = check_part(Vs, sVs, B, Hkv, S, d, false, &p.mvs)) != SPARK_OK) return rc;
  if ((rc = check_part(O, sO, B, H, Nq, d, false, &p.mo)) != SPARK_OK) return rc;
  if ((rc = check_part(dO, sdO, B, H, Nq, d, false, &a.mdo)) != SPARK_OK) return rc;
  if ((rc = check_part(dQ, sdQ, B, H, Nq, d, true, &a.mdq)) != SPARK_OK) return rc;
  if ((rc = check_part(dKp, sdKp, G, Hkv, P, d, true, &a.mdkp)) != SPARK_OK) return rc;
  if ((rc = check_part(dVp, sdVp, G, Hkv, P, d, true, &a.mdvp)) != SPARK_OK) return rc;
  if ((rc = check_part(dKs, sdKs, B, Hkv, S, d, true, &a.mdks)) != SPARK_OK) return rc;
  if ((rc = check_part(dVs, sdVs, B, Hkv, S, d, true, &a.mdvs)) != SPARK_OK) return rc;
  if (!aligned16(LSE) || !aligned16(workspace)) return SPARK_ERR_ALIGN;
  if (workspace_bytes < prefix_bwd_workspace(p)) return SPARK_ERR_WORKSPACE;
  p.Q = Q; p.Kp = Kp; p.Vp = Vp; p.Ks = Ks; p.Vs = Vs;
  p.prefix_lens = prefix_lens; p.q_lens = q_lens; p.s_lens = s_lens;
  a.dO = dO; a.dQ = dQ; a.dKp = dKp; a.dVp = dVp; a.dKs = dKs; a.dVs = dVs; a.LSE = LSE; a.workspace = workspace;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == SPARK_F16 ? dispatch_prefix_bwd<_Float16>(p, O, a, scale, st)
                            : dispatch_prefix_bwd<__bf16>(p, O, a, scale, st);
}

size_t spark_mha_prefix_fwd_workspace_bytes(int G, int B, int H, int Hkv, int Nq, int P, int S, int d, spark_dtype_t dtype) {
  PrefixProblem p{};
  if (make_prefix(&p, G, B, H, Hkv, Nq, P, S, d, 1.0f, 0, (int)dtype) != SPARK_OK) return 0;
  return prefix_fwd_workspace(p);
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
  if (workspace && workspace_bytes < prefix_fwd_workspace(p)) return SPARK_ERR_WORKSPACE;
  p.Q = Q; p.Kp = Kp; p.Vp = Vp; p.Ks = Ks; p.Vs = Vs;
  p.prefix_lens = prefix_lens; p.q_lens = q_lens; p.s_lens = s_lens;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == SPARK_F16 ? dispatch_prefix_fwd<_Float16>(p, O, LSE, workspace, scale, st)
                            : dispatch_prefix_fwd<__bf16>(p, O, LSE, workspace, scale, st);
}

}  // extern "C"
