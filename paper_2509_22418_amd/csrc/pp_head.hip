// Losses of the output head (cross entropy, distillation from a teacher's top logits) with their gradients, the logits existing a piece of rows at a time.
//
// With z = X W^T:  dz_tv = g_t [ c1 (p_tv - [v = y_t]) + ct (pt_tv - Q_tv) ],  p = softmax(z), pt = softmax(z / tau), c1 = 1 - share (rows with a target), ct = share tau (rows
// with entries), Q the teacher's q at its entries;  dX = dz W,  dW = dz^T X.
// Rows that count are gathered into the front of the workspace's copy of X, whose rows are padded with zeros to what the matrix kernels read; every
// kernel below works on those compact rows, in pieces.
//
// bf16: the first product's epilogue stores e = exp((z - r) / tau) instead of z, r a reference of the row that is known BEFORE the product: the largest logit among the target's and
// the teacher's entries.  A softmax needs no more of its reference than that no exponential overflows or is lost, so the maximum itself is not waited for, and e's rounding to bf16
// is relative.  With s = sum e the row of dz is a multiple of e but for the target and the entries:
//     dz = g C (e - sub / C),  C = c / s,  sub = c1 [v = y] + ct Q,  g the row's weight:
// a kernel over rows replaces e at those few places, and g C is applied to dX's rows behind their product and to X's rows in front of dW's.  No other pass over the piece, and no second
// product of logits: 2 products for dX alone, 3 with dW.  Rows whose largest logit turns out to lie more than kFar from the reference take the maximum, and the first product of
// their 256-row blocks is done again (by a launch that ends at once where there are none).  Two softmaxes at once (tau != 1 beside hard targets) take one more pass
// over the piece, which forms both exponentials from the one exponent that the first product then stores.
// Pieces are of rows, not of the vocabulary: a piece of vocabulary would have to wait for the sums of all others, hence form its logits twice (4 products instead of 3), and sum dX in
// memory.  fp32: logits in fp32, softmax and dz by a block per row, products on the fp32 MFMA kernels.
#include "pp_kernels.h"
#include "pp_dev.h"

#include <algorithm>

namespace pp {

#define PP_H_DISPATCH(dtype, ...)                                       \
  do {                                                                  \
    if ((dtype) == 0) { using T = float; __VA_ARGS__; }                 \
    else { using T = bf16_t; __VA_ARGS__; }                             \
  } while (0)

// ------------------------------------------------------------------------------------------------ plan
namespace {
constexpr int kTopMax = 128;          // entries per row (PP_HEAD_TOP_MAX)
constexpr size_t kPieceBytes = 512ull << 20;
struct HeadPlan {
  int dp, vp, np, piece, groups, exp_tile;          // padded width, padded vocabulary, rows of the compact X, rows of a piece, column groups of the first product's partial sums, its tile (0: 256)
  int dx_splits, dw_splits, n_redo, ref_group, parts;          // ref_group: entries per wave of head_ref_kernel; parts: waves of the first product of few rows (0: the other kernels)
  bool grads, copy_w, own_wt, mixed, dx_whole, pick;          // pick: the first product picks the entries' logits
  size_t flags, pos, rows, count, rowl, ref, scale, coef, zsel, xc, wc, wt, z, stats, stats2, redo, offs, list, xt, part, dwa, total;          // byte offsets
};
int pad_to(long v, int m) { return (int)((v + m - 1) / m * m); }

// K ranges of a product of `tiles` 256 x 256 tiles and `steps` steps of 64: the number that fills rounds of 256 workgroups best.  In 1 / 4 us: a step takes 1.6 us, a workgroup 10 us besides (30 with
// partial sums to write), and the launch that sums them 5 us and 0.1 us per tile and range.  (32000 x 768 over 8192 rows, 375 tiles: one range 415 us, two 397 + 73; 8192 x 768 over 32000,
// 96 tiles: two 412 + 14, five 402 + 28; 3277 x 2048 over 32000, 104 tiles: one 572, two 345 + 26.)
constexpr int kMaxSplits = 32;
__host__ __device__ inline int splits_cost(int tiles, int steps, int s) {
  return (tiles * s + 255) / 256 * ((steps + s - 1) / s * 32 / 5 + (s > 1 ? 120 : 40)) + (s > 1 ? 20 + s * tiles * 2 / 5 : 0);
}
int best_splits(int tiles, int steps, int most) {
  int best = 1;
  for (int s = 2; s <= most && steps >= 8 * s && tiles <= 1024; ++s)
    if (splits_cost(tiles, steps, s) < splits_cost(tiles, steps, best)) best = s;
  return best;
}
// ranges that fit the buffer of the partial sums
int capped(int splits, double mn, size_t cap) {
  while (splits > 1 && cap && splits * mn * 4 > (double)cap) --splits;
  return splits;
}

// Few rows: threads of a workgroup side by side (8 columns each), and rows of W per workgroup such that the workgroups' partial sums of dX are kFewPartials at most.
constexpr int kFew = 16, kFewPartials = 512;
// Small vocabularies of long rows: the four waves of a workgroup take a quarter of 16 rows of W each (2 rows of X, 5280 x 3999 in fp32: 70 -> 45 us)
bool few_split(int tiles, int d) { return tiles <= 512 && d > 256; }
int few_cols(int d) { int c = 1; while (c < 256 && c * 8 < d) c *= 2; return c; }
int few_waves(int d) { return d > 256 ? 4 : d > 128 ? 2 : 1; }          // waves side by side where dX and dW are formed by MFMAs, 128 columns each (from two rows on: 4 x 2048 x 32000 dX 74 -> 71 us, 16 x 768 69 -> 56; one row has too little to multiply)
// rows of W per workgroup of dX: one row of X (vector units) two for every thread at least; more rows (MFMAs) as many as make 1024 workgroups with the column slices
int few_chunk(int rows, int d, int n) {
  if (n == 1) return std::max((rows + kFewPartials - 1) / kFewPartials, 2 * 256 / few_cols(d));
  const int slice = few_waves(d) * 128, groups = std::max(1, std::min(kFewPartials, 1024 / ((d + slice - 1) / slice)));
  return std::max((rows + groups - 1) / groups, 32);
}

HeadPlan plan_head(const HeadArgs& a) {
  HeadPlan p{};
  const bool bf = a.dtype != 0;
  const size_t es = bf ? 2 : 4;
  const int unit = bf ? 64 : 128;          // fp32: dX's contraction in up to 32 ranges of whole groups of four
  const int dw_rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  p.grads = a.dx || a.dw;
  p.mixed = a.tau != 1.f && a.share > 0.f && a.share < 1.f;
  p.dp = pad_to(a.d, bf ? 64 : 4);
  p.vp = pad_to(a.vocab, unit);
  p.np = std::max(64, pad_to(a.n, 64));
  if (a.n > 0 && a.n <= kFew && !a.no_few) {
    // up to 2048 waves, 8 a compute unit, each with as many of the blocks of 16 rows of W as any other
    const int tiles = (a.vocab + 15) / 16, each = (tiles + 2047) / 2048;
    p.parts = ((tiles + each - 1) / each + 3) / 4 * 4;
    if (few_split(tiles, a.d)) p.parts = 4 * tiles;
    p.vp = pad_to(a.vocab, 16);
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off += (bytes + 255) / 256 * 256; return o; };
    p.rowl = take(kFew * 4);
    p.z = take((size_t)a.n * p.vp * 4);
    p.stats = take((size_t)kFew * (p.parts / 4) * 16);
    p.coef = take(kFew * 16);
    p.scale = take((size_t)kFew * (a.top + 1) * 4);
    p.zsel = take((size_t)kFew * (a.top + 1) * 4);
    if (a.dx) {
      const int chunk = few_chunk(a.vocab, a.d, a.n);
      p.part = take((size_t)((a.vocab + chunk - 1) / chunk) * a.n * a.d * 4);
    }
    p.total = off;
    return p;
  }
  const size_t row = (size_t)p.vp * es;
  // Every piece but the first reads and writes dW's fp32 sums: with a larger dW the pieces may be as large as that, up to 1 GiB (4096 x 4096 x 128000, in two pieces / in one: 10.5 / 9.5 ms)
  const size_t limit = std::max(kPieceBytes, std::min(2 * kPieceBytes, (size_t)dw_rows * a.d * 4));
  p.piece = a.piece ? pad_to(a.piece, 64) : std::max(256, (int)(limit / row / 256 * 256));
  // 2^18: grids of piece / 64 in y.  2 GiB: the products' 32-bit offsets and whatever a caller asks for
  p.piece = std::min({p.piece, p.np, 1 << 18, std::max(256, (int)((2ull << 30) / row / 256 * 256))});
  if (bf) {
    // The first product's tiles, and the logits of the teacher's entries: by dot products (head_ref_kernel: a row of W each, 7 TB/s out of the last-level cache, half a microsecond for each of a
    // wave's ref_group), or picked from the accumulators of 256 x 256 tiles (the lists, and their look-ups in every tile; 8192 x 2048 x 32000 with 64 entries a row 315 us / 50 us).  The estimates,
    // in us, are fitted to 165 shapes timed both ways (widths of 256 to 2048, 700 to 8000 rows, vocabularies of 8000 to 100000, 2 to 64 entries): on 159 the faster or one within 3 % of it is
    // taken, on the others one within 7 %.  The last piece, which may be smaller, takes the tiles of the others.
    // More waves with fewer entries each, where all rows' groups of 16 would be less than four waves a compute unit.
    p.ref_group = 16;
    while (p.ref_group > 4 && (long)p.np * ((a.top + p.ref_group - 1) / p.ref_group) < 1024) p.ref_group /= 2;
    const double big = head_exp_us(p.piece, a.vocab, p.dp, 0), t128 = head_exp_us(p.piece, a.vocab, p.dp, 128), t64 = head_exp_us(p.piece, a.vocab, p.dp, 64);
    const double rounds = (double)((p.piece + 255) / 256) * ((a.vocab + 255) / 256) / 256;
    const double dots = a.top ? (double)p.piece * a.top * p.dp * 2 / 7e6 + std::min(a.top, p.ref_group) / 2. : 0;
    const double picked = a.top && a.vocab <= 1 << 19 ? 6 + a.top / 12. + rounds * a.vocab / 9e4 : 1e30;          // (the lists' counters fit 32 KB of LDS)
    p.pick = big + picked < std::min({big, t128, t64}) + dots;
    p.exp_tile = p.pick || std::min(t128, t64) >= big ? 0 : t64 < t128 ? 64 : 128;
  }
  const int wide = p.exp_tile ? p.exp_tile : 256;          // columns that one partial sum of a row covers, by the tiles
  p.groups = (a.vocab + wide - 1) / wide * (wide / (p.exp_tile ? 32 : 64));
  // the bf16 matrix kernels read rows that are multiples of 64 elements long, 16-byte aligned and not so far apart that the offsets among 64 of them pass 31 bits; the fp32 ones any
  p.copy_w = bf && (a.d % 64 || a.ldw % 8 || a.ldw > 1 << 22 || (uintptr_t)a.w & 15);
  p.own_wt = a.dx && !bf && !(a.wt && a.vocab % unit == 0);          // the bf16 products read W as it lies
  // dX's ranges are decided on the device by the rows that count (head_scan_kernel): at most so many, and partial sums for the worst number of rows
  const int tiles_d = (a.d + 255) / 256;
  size_t dx_part = 0;
  p.dx_splits = 1;
  p.dx_whole = (p.piece + 255) / 256 * tiles_d > 1024;          // whether any number of rows takes one range
  if (bf && a.dx)
    for (int t = 1; t <= (p.piece + 255) / 256 && t * tiles_d <= 1024; ++t) {
      const size_t rows = std::min(t * 256, p.piece);
      const int s = capped(best_splits(t * tiles_d, p.vp / 64, kMaxSplits), (double)rows * a.d, a.part_cap);
      p.dx_splits = std::max(p.dx_splits, s);
      p.dx_whole |= s == 1;
      if (s > 1) dx_part = std::max(dx_part, s * rows * a.d * 4);
    }
  p.dw_splits = bf && a.dw ? capped(best_splits((dw_rows + 255) / 256 * tiles_d, p.piece / 64, kMaxSplits), (double)dw_rows * a.d, a.part_cap) : 1;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += (bytes + 255) / 256 * 256; return o; };
  p.flags = take(a.top ? p.np : 0);
  p.pos = take((size_t)p.np * 4);
  p.rows = take((size_t)p.np * 4);
  p.count = take(256);
  p.rowl = take((size_t)p.np * 4);
  p.xc = take((size_t)p.np * p.dp * es);
  p.wc = take(p.copy_w ? (size_t)a.vocab * p.dp * es : 0);
  p.wt = take(p.own_wt ? (size_t)a.d * p.vp * es : 0);
  if (bf) {
    p.ref = take((size_t)p.np * 4);
    p.scale = take((size_t)p.np * 4);
    p.coef = take(a.top ? (size_t)p.piece * 8 : 0);
    p.zsel = take((size_t)p.np * (a.top + 1) * 4);
    p.z = take(p.grads ? (size_t)p.piece * p.vp * es : 0);
    const size_t sums = (size_t)(a.part_cap ? (a.vocab + 255) / 256 * 8 : p.groups) * p.piece;          // part_cap: for either tile, so that fewer rows never need more
    p.stats = take(sums * 8);
    p.stats2 = take(a.top ? sums * 4 : 0);          // temperature and share are not known where the size is asked for
    const int pieces = (p.np + p.piece - 1) / p.piece;
    p.n_redo = pieces * (1 + (p.piece + 255) / 256);
    p.redo = take((size_t)(p.n_redo + pieces) * 4);          // then the ranges of every piece's dX
    const bool room = p.pick || (a.part_cap && a.top);          // part_cap: fewer entries or rows never need more
    p.offs = take(room ? (size_t)(p.piece + 127) / 128 * ((a.vocab + 255) / 256 * 4 + 1) * 4 : 0);
    p.list = take(room ? (size_t)(p.piece + 127) / 128 * 128 * a.top * 4 : 0);
    p.xt = take(a.dw ? (size_t)a.d * p.piece * es : 0);
    p.part = take(a.part_cap ? a.part_cap : std::max(dx_part, p.dw_splits > 1 ? (size_t)p.dw_splits * dw_rows * a.d * 4 : 0));
    p.dwa = take(a.dw && !a.dw_f32 && p.piece < a.n ? (size_t)dw_rows * a.d * 4 : 0);
  } else {
    // ranges of the contractions: doubled until the products have two workgroups of 64 x 64 tiles for a compute unit (1024 x 512, K = 8000: one range of 32 x 32 tiles 94 us)
    auto double_up = [&](long tiles, int k, int unit_k, size_t out) {
      int s = 1;
      while (s < 32 && tiles * s < 512 && k % (2 * s * unit_k) == 0 && k / (2 * s) >= 512 && (!a.part_cap || 2 * s * out <= a.part_cap)) s *= 2;
      return s;
    };
    const long t64 = (a.d + 63) / 64;
    p.dx_splits = a.dx ? double_up((p.piece + 63) / 64 * t64, p.vp, 4, (size_t)p.piece * a.d * 4) : 1;
    p.dw_splits = a.dw ? double_up((dw_rows + 63) / 64 * t64, p.piece, 4, (size_t)dw_rows * a.d * 4) : 1;
    p.z = take((size_t)p.piece * p.vp * 4);
    p.part = take(std::max({a.part_cap, a.dx ? (size_t)p.dx_splits * p.piece * a.d * 4 : (size_t)0, p.dw_splits > 1 || p.piece < a.n || a.dw_f32 == 2 ? (size_t)p.dw_splits * dw_rows * a.d * 4 : (size_t)0}));
  }
  p.total = off;
  return p;
}
}  // namespace
size_t head_bytes(const HeadArgs& a) { return plan_head(a).total; }
bool head_is_few(const HeadArgs& a) { return plan_head(a).parts > 0; }

// ------------------------------------------------------------------------------------------------ rows that count
enum { ROW_HARD = 1, ROW_SOFT = 2 };
__device__ __forceinline__ bool hard_row(const int32_t* targets, int t, int V) { return targets && (uint32_t)targets[t] < (uint32_t)V; }

// distillation: which terms a row has, a wave per row
__global__ __launch_bounds__(256) void head_flags_kernel(const int32_t* __restrict__ targets, const int32_t* __restrict__ ids, const float* __restrict__ logits, const float* __restrict__ weight,
                                                         unsigned char* __restrict__ flags, int n, int V, int top, int use_soft) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= n) return;
  bool there = false;
  if (use_soft)
    for (int j = lane; j < top; j += 64) there |= (uint32_t)ids[(size_t)t * top + j] < (uint32_t)V && logits[(size_t)t * top + j] != -INFINITY;
  const bool soft = __ballot(there) != 0;
  if (lane == 0) flags[t] = weight && weight[t] == 0.f ? 0 : (hard_row(targets, t, V) ? ROW_HARD : 0) | (soft ? ROW_SOFT : 0);
}

// pos[t] = place of row t among the rows that count, -1 for the others; rows[i] = t; count = their number; redo cleared.  One block, 16 rows per thread at a time: rows 1024 apart, so that
// what a wave reads and writes lies together.
__global__ __launch_bounds__(1024) void head_scan_kernel(const int32_t* __restrict__ targets, const unsigned char* __restrict__ flags, const float* __restrict__ weight, int n, int V,
                                                         int32_t* __restrict__ pos, int32_t* __restrict__ rows, int32_t* __restrict__ count, int32_t* __restrict__ redo, int n_redo, int pieces, int piece,
                                                         int tiles_d, int steps, int most, size_t cap, int d) {
  __shared__ int total_s, part_s[256];          // rows that count of wave w in the e-th 1024 at [16 e + w]; then those before them
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < n_redo; i += 1024) redo[i] = 0;
  int base = 0;
  for (int t0 = 0; t0 < n; t0 += 16 * 1024) {
    uint32_t live = 0;
    int32_t y[16];          // all of a thread's loads in flight, from clamped places
    float g[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      y[e] = -1;
      g[e] = 1.f;
      if (t0 + e * 1024 >= n) continue;
      const int t = min(t0 + e * 1024 + tid, n - 1);
      y[e] = flags ? flags[t] : targets[t];
      if (weight && !flags) g[e] = weight[t];
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (t0 + e * 1024 + tid < n && (flags ? y[e] != 0 : (uint32_t)y[e] < (uint32_t)V && g[e] != 0.f)) live |= 1u << e;
    uint64_t ballot[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      ballot[e] = __ballot(live >> e & 1);
      if (lane == 0) part_s[16 * e + wave] = __popcll(ballot[e]);
    }
    __syncthreads();
    if (wave == 0) {          // exclusive sums of the 256 parts, four per lane
      int v[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) { v[k] = part_s[4 * lane + k]; sum += v[k]; }
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(incl, o, 64);
        if (lane >= o) incl += u;
      }
      int before = incl - sum;
#pragma unroll
      for (int k = 0; k < 4; ++k) { part_s[4 * lane + k] = before; before += v[k]; }
      if (lane == 63) total_s = before;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int t = t0 + e * 1024 + tid, at = base + part_s[16 * e + wave] + __popcll(ballot[e] & ((1ull << lane) - 1));
      if (t >= n) continue;
      const bool l = live >> e & 1;
      pos[t] = l ? at : -1;
      if (l) rows[at] = t;
    }
    base += total_s;
    __syncthreads();
  }
  if (tid == 0) *count = base;
  for (int i = wave; i < pieces; i += 16) {          // every piece's ranges of dX's contraction (best_splits), a number of ranges per lane
    const int live = min(max(base - i * piece, 0), piece), rows = (live + 63) & ~63, mine = lane + 1;
    static_assert(kMaxSplits <= 64, "a lane each");
    const int cost = splits_cost((live + 255) / 256 * tiles_d, steps, mine);
    const bool can = mine == 1 || (mine <= most && steps >= 8 * mine && (live + 255) / 256 * tiles_d <= 1024);
    int low = can ? cost : 0x7fffffff;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) low = min(low, __shfl_xor(low, o, 64));
    int s = __ffsll((unsigned long long)__ballot(can && cost == low));
    while (s > 1 && cap && (double)s * rows * d * 4 > (double)cap) --s;
    if (lane == 0) redo[n_redo + i] = s;
  }
}

// columns c .. c + 3 of a row of d, those there are
__device__ __forceinline__ float4 load_cols(const float* row, int c, int d) {
  if (c + 4 <= d) {
    const any16 r = *reinterpret_cast<const any16*>(row + c);
    return make_float4(__uint_as_float(r.w[0]), __uint_as_float(r.w[1]), __uint_as_float(r.w[2]), __uint_as_float(r.w[3]));
  }
  return make_float4(c < d ? row[c] : 0.f, c + 1 < d ? row[c + 1] : 0.f, c + 2 < d ? row[c + 2] : 0.f, 0.f);
}
__device__ __forceinline__ void store_cols(float* row, int c, int d, const float4& v) {
  if (c + 4 <= d) *reinterpret_cast<any16*>(row + c) = any16{{__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)}};
  else {
    if (c < d) row[c] = v.x;
    if (c + 1 < d) row[c + 1] = v.y;
    if (c + 2 < d) row[c + 2] = v.z;
  }
}
__device__ __forceinline__ void store_cols(bf16_t* row, int c, int d, const float4& v) {
  if (c + 4 <= d) *reinterpret_cast<any8*>(row + c) = any8{{f32x2_to_bf16x2(v.x, v.y), f32x2_to_bf16x2(v.z, v.w)}};
  else {
    if (c < d) row[c] = from_f32<bf16_t>(v.x);
    if (c + 1 < d) row[c + 1] = from_f32<bf16_t>(v.y);
    if (c + 2 < d) row[c + 2] = from_f32<bf16_t>(v.z);
  }
}

// Compact, padded copy of the rows that count; zeros behind them up to the last row of the copy; the outputs of rows that are left out.  A wave per row.
__global__ __launch_bounds__(256) void head_gather_kernel(const float* __restrict__ x, int ldx, float* __restrict__ xc, int dp, int d, const int32_t* __restrict__ pos, const int32_t* __restrict__ count,
                                                          int n, int np, float* __restrict__ dx, int lddx, float* __restrict__ row_loss, float* __restrict__ row_lse) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= np) return;
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  if (t >= *count)
    for (int c = 4 * lane; c < dp; c += 256) *reinterpret_cast<float4*>(xc + (size_t)t * dp + c) = zero;
  if (t >= n) return;
  const int i = pos[t];
  if (i < 0) {
    if (dx) for (int c = 4 * lane; c < d; c += 256) store_cols(dx + (size_t)t * lddx, c, d, zero);
    if (lane == 0) { row_loss[t] = 0.f; if (row_lse) row_lse[t] = 0.f; }
    return;
  }
#pragma unroll 4
  for (int c = 4 * lane; c < dp; c += 256) *reinterpret_cast<float4*>(xc + (size_t)i * dp + c) = load_cols(x + (size_t)t * ldx, c, d);
}

// dst [rows x ld_dst] = src [rows x cols], zeros from column cols to ld_dst, a multiple of 8; dst 16-byte aligned.  A wave per row.
__global__ __launch_bounds__(256) void head_pad_kernel(const bf16_t* __restrict__ src, int ld_src, bf16_t* __restrict__ dst, int ld_dst, int rows, int cols) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const bf16_t* from = src + (size_t)r * ld_src;
#pragma unroll 4
  for (int c = (threadIdx.x & 63) * 8; c < ld_dst; c += 512) {
    uint4 v;
    if (c + 8 <= cols) {
      const any16 u = *reinterpret_cast<const any16*>(from + c);
      v = make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = c + k < cols ? from[c + k].bits : 0;
      v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
    *reinterpret_cast<uint4*>(dst + (size_t)r * ld_dst + c) = v;
  }
}
// dst[c][r] = src[r][c] for r < rows, zeros for rows <= r < ld_dst
template <class T>
__global__ __launch_bounds__(256) void head_transpose_kernel(const T* __restrict__ src, int ld_src, T* __restrict__ dst, int ld_dst, int rows, int cols) {
  __shared__ T tile[64][65];
  const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  T v[16];          // all rows of a thread requested at once, from clamped addresses
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = src[(size_t)min(r0 + ty + 4 * k, rows - 1) * ld_src + min(c0 + tx, cols - 1)];
#pragma unroll
  for (int k = 0; k < 16; ++k) tile[ty + 4 * k][tx] = r0 + ty + 4 * k < rows ? v[k] : from_f32<T>(0.f);
  __syncthreads();
  for (int i = ty; i < 64; i += 4)
    if (c0 + i < cols && r0 + tx < ld_dst) dst[(size_t)(c0 + i) * ld_dst + r0 + tx] = tile[tx][i];
}

// ------------------------------------------------------------------------------------------------ softmax, losses and dz of a row of logits
// One block per compact row of the piece: z [piece x vp] fp32 becomes dz (columns behind the vocabulary zero) if `grads`.
struct HeadRow {
  const int32_t *rows, *count, *targets, *ids;
  const float *logits, *weight;
  const unsigned char* flags;
  float *row_loss, *row_lse;
  float tau, share;
  int V, vp, top, i0;
};
// The row's entries in shared memory: q[j] of entry j (0 where there is none) and its id (-1).  Every thread calls it.
__device__ __forceinline__ void head_entries(const HeadRow& h, int t, int* id_s, float* q_s, float* red) {
  const int j = threadIdx.x;
  int id = -1;
  float u = -INFINITY;
  if (j < h.top) {
    id = h.ids[(size_t)t * h.top + j];
    if ((uint32_t)id < (uint32_t)h.V) u = h.logits[(size_t)t * h.top + j]; else id = -1;
    if (u == -INFINITY) id = -1;
  }
  // NaN among the entries has to reach the sum: fmaxf would drop it from the maximum
  const float m = block_max(id >= 0 ? u : -INFINITY, red);
  const float e = id >= 0 ? expf((u - m) / h.tau) : 0.f;          // the largest first: the lowest finite value over a low temperature is not finite
  const float s = block_sum(e, red);
  if (j < h.top) { id_s[j] = id; q_s[j] = id >= 0 ? e / s : 0.f; }
  __syncthreads();
}

// BS threads, NV groups of four logits a thread held in registers (0: the row is read for the sums and again for dz; 16 groups would spill).  One read and one write of the row where it fits.
template <int BS, int NV>
__global__ __launch_bounds__(BS) void head_row_kernel(float* z_, int grads, HeadRow h) {
  __shared__ float red[17];
  __shared__ int id_s[kTopMax];
  __shared__ float q_s[kTopMax];
  const int i = h.i0 + blockIdx.x, tid = threadIdx.x, n_live = *h.count;
  if (i >= n_live) return;          // nothing reads these rows
  float* z = z_ + (size_t)blockIdx.x * h.vp;
  const int t = h.rows[i], groups = h.vp / 4;
  const bool hard = h.flags ? h.flags[t] & ROW_HARD : true, soft = h.flags ? h.flags[t] & ROW_SOFT : false;
  const float it = 1.0f / h.tau;
  constexpr int KEEP = NV > 0 ? NV : 1;
  float4 r[KEEP];
  auto fetch = [&](int g) {          // columns behind the vocabulary as -inf
    float4 v = g < groups ? *reinterpret_cast<const float4*>(z + 4 * g) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (4 * g + 4 > h.V) { if (4 * g >= h.V) v.x = -INFINITY; if (4 * g + 1 >= h.V) v.y = -INFINITY; if (4 * g + 2 >= h.V) v.z = -INFINITY; v.w = -INFINITY; }
    return v;
  };
  auto each = [&](auto f) {          // f(group index, its four logits)
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) f(tid + BS * k, r[k]);
    } else
      for (int g = tid; g < groups; g += BS) f(g, fetch(g));
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) r[k] = fetch(tid + BS * k);
  }
  float m = -INFINITY, s1 = 0.f, st = 0.f;
  const bool two = h.tau != 1.f;
  auto sums = [&](const float4& v, float top) {
    s1 += expf(v.x - top) + expf(v.y - top) + expf(v.z - top) + expf(v.w - top);
    if (two) st += expf((v.x - top) * it) + expf((v.y - top) * it) + expf((v.z - top) * it) + expf((v.w - top) * it);
  };
  auto largest = [](float m, const float4& v) { return fmaxf(fmaxf(m, fmaxf(v.x, v.y)), fmaxf(v.z, v.w)); };
  if constexpr (NV > 0) {
    each([&](int, const float4& v) { m = largest(m, v); });
    m = block_max(m, red);
    each([&](int, const float4& v) { sums(v, m); });
  } else {          // one read for both: a thread's sums are against the largest logit it has seen
    float mine = -INFINITY;
    each([&](int, const float4& v) {
      const float top = largest(mine, v);
      if (top > mine) {
        s1 *= expf(mine - top);
        if (two) st *= expf((mine - top) * it);
        mine = top;
      }
      if (mine != -INFINITY) sums(v, mine);
      else s1 += v.x + v.y + v.z + v.w != -INFINITY ? NAN : 0.f;          // nothing but -inf and NaN so far: NaN has to reach the sum
    });
    m = block_max(mine, red);
    const float back = mine == -INFINITY ? 1.f : expf(mine - m);
    s1 *= back;
    if (two) st *= mine == -INFINITY ? 1.f : expf((mine - m) * it);
  }
  s1 = block_sum(s1, red);
  st = two ? block_sum(st, red) : s1;
  if (soft) head_entries(h, t, id_s, q_s, red);
  const int y = hard ? h.targets[t] : -1;
  // losses
  float kl = 0.f;
  if (soft && tid < h.top && id_s[tid] >= 0 && !(q_s[tid] <= 0.f)) kl = q_s[tid] * (logf(q_s[tid]) - (z[id_s[tid]] - m) * it + logf(st));
  if (h.top) kl = block_sum(kl, red);
  if (tid == 0) {
    float l = soft ? h.share * h.tau * h.tau * kl : 0.f;
    if (hard) l += (1.f - h.share) * ((m - z[y]) + logf(s1));
    h.row_loss[t] = l;
    if (h.row_lse) h.row_lse[t] = m * it + logf(st);
  }
  if (!grads) return;
  const float g = h.weight ? h.weight[t] : 1.0f / (float)n_live;
  const float c1 = hard ? g * (1.f - h.share) : 0.f, ct = soft ? g * h.share * h.tau : 0.f;
  const float p1 = c1 / s1, pt = ct / st;
  auto soft_part = [&](float zv) { return (c1 != 0.f ? p1 * expf(zv - m) : 0.f) + (ct != 0.f ? pt * expf((zv - m) * it) : 0.f); };
  // entry j of the row, or the target (j == top): its part of dz is formed from z before dz takes its place.  The first of equal ids stores the sum of all, in their order.
  float own = 0.f;
  int at = -1;
  if (tid <= h.top) {
    at = tid < h.top ? (soft ? id_s[tid] : -1) : y;
    if (at >= 0) {
      float sub = 0.f;
      bool first = true;
      if (soft)
        for (int k = 0; k < h.top; ++k)
          if (id_s[k] == at) { if (k < tid) first = false; sub += ct * q_s[k]; }
      if (at == y) sub += c1;
      if (first) own = soft_part(z[at]) - sub; else at = -1;
    }
  }
  __syncthreads();
  each([&](int gi, const float4& v) { if (gi < groups) *reinterpret_cast<float4*>(z + 4 * gi) = make_float4(soft_part(v.x), soft_part(v.y), soft_part(v.z), soft_part(v.w)); });
  __syncthreads();
  if (at >= 0) z[at] = own;
}

// ------------------------------------------------------------------------------------------------ bf16: references, sums, losses and the places that differ
// What head_gather_kernel does, and for the rows that count zsel[i][j] = z of entry j of compact row i (j == top: of its target) by a wave's dot products in fp32 and ref[i] = the largest of
// them (0 behind the last row that counts).  xc and w rows are dp (a multiple of 64) elements, 16-byte aligned.
struct HeadRef {
  const bf16_t *x, *w;
  bf16_t *xc, *dx;
  int ldx, ldw, lddx, d, dp, n, np, V, top, vec, group;          // vec: rows of x are whole aligned groups of 8; group: entries per blockIdx.y, 1: the first one only
  const int32_t *pos, *count, *targets, *ids;
  const float* logits;
  const unsigned char* flags;
  float *zsel, *ref, *row_loss, *row_lse;
};
__global__ __launch_bounds__(256) void head_ref_kernel(HeadRef h) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= h.np) return;
  if (t >= *h.count && blockIdx.y == 0) {
    for (int c = lane * 8; c < h.dp; c += 512) *reinterpret_cast<uint4*>(h.xc + (size_t)t * h.dp + c) = make_uint4(0, 0, 0, 0);
    if (lane == 0) h.ref[t] = 0.f;
  }
  if (t >= h.n) return;
  const int i = h.pos[t];
  if (i < 0) {
    if (blockIdx.y) return;
    if (h.dx) for (int c = lane; c < h.d; c += 64) h.dx[(size_t)t * h.lddx + c] = from_f32<bf16_t>(0.f);
    if (lane == 0) { h.row_loss[t] = 0.f; if (h.row_lse) h.row_lse[t] = 0.f; }
    return;
  }
  const bool hard = h.flags ? h.flags[t] & ROW_HARD : true, soft = h.flags ? h.flags[t] & ROW_SOFT : false;
  const bf16_t* x = h.x + (size_t)t * h.ldx;
  bf16_t* xc = h.xc + (size_t)i * h.dp;
  float* zs = h.zsel + (size_t)i * (h.top + 1);
  float best = -INFINITY;
  // Entries in groups over blockIdx.y (the first entry alone, group 1, where the first product picks all logits), the target (entry `top`) and the row's copy with the first; the reference is the largest of that first group,
  // or the row's first entry where the group has none and the row no target: a reference far above all logits would lose every exponential.
  constexpr int NB = 8;          // entries at a time: eight rows of W in flight
  int lo = blockIdx.y * h.group, hi = soft ? min(lo + h.group, h.top) : lo;
  auto first_entry = [&]() {          // the first entry there is, -1 if none is
    for (int j = 0; j < h.top; j += 64) {
      const bool is = j + lane < h.top && (uint32_t)h.ids[(size_t)t * h.top + j + lane] < (uint32_t)h.V && h.logits[(size_t)t * h.top + j + lane] != -INFINITY;
      if (const uint64_t there = __ballot(is)) return j + (int)__ffsll((unsigned long long)there) - 1;
    }
    return -1;
  };
  if (h.group == 1 && soft) {
    const int j = first_entry();
    if (j >= 0) { lo = j; hi = j + 1; }
  }
  if (blockIdx.y && lo >= hi) return;
  const int list = hi - lo + (blockIdx.y == 0);          // entries of this wave, the target last
  for (int k0 = 0; k0 < list; k0 += NB) {
    int id[NB];
    float s[NB];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
      const int j = lo + k0 + e, v = j < hi ? h.ids[(size_t)t * h.top + j] : j == hi && blockIdx.y == 0 && hard ? h.targets[t] : -1;
      const float uj = j < hi ? h.logits[(size_t)t * h.top + j] : 0.f;
      id[e] = (uint32_t)v < (uint32_t)h.V && uj != -INFINITY ? v : -1;
      s[e] = 0.f;
    }
    const bool copy = blockIdx.y == 0 && k0 == 0;
    for (int c = lane * 8; c < h.dp; c += 512) {
      uint4 raw;
      if (h.vec && c + 8 <= h.d) raw = *reinterpret_cast<const uint4*>(x + c);
      else {
        uint16_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < h.d ? x[c + k].bits : (uint16_t)0;
        raw = make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
      }
      if (copy) *reinterpret_cast<uint4*>(xc + c) = raw;
      const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
      float xv[8], wv[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) { xv[2 * k] = __uint_as_float(rw[k] << 16); xv[2 * k + 1] = __uint_as_float(rw[k] & 0xffff0000u); }
#pragma unroll
      for (int e = 0; e < NB; ++e)
        if (id[e] >= 0) {
          load8(h.w + (size_t)id[e] * h.ldw + c, wv);
#pragma unroll
          for (int k = 0; k < 8; ++k) s[e] = fmaf(xv[k], wv[k], s[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < NB; ++e)
      if (id[e] >= 0) {
        const float z = wave_sum(s[e]);
        if (lane == 0) zs[lo + k0 + e == hi ? h.top : lo + k0 + e] = z;
        best = fmaxf(best, z);
      }
  }
  if (blockIdx.y) return;
  if (soft && best == -INFINITY) {          // no target, and nothing in the first group: the first entry there is, whose dot product another wave forms too
    const int j = first_entry();
    float s = 0.f;
    if (j >= 0) {
      const bf16_t* w = h.w + (size_t)h.ids[(size_t)t * h.top + j] * h.ldw;
      for (int c = lane * 8; c < h.dp; c += 512) {
        float xv[8], wv[8];
        load8(xc + c, xv);          // this lane's own stores
        load8(w + c, wv);
#pragma unroll
        for (int k = 0; k < 8; ++k) s = fmaf(xv[k], wv[k], s);
      }
      best = wave_sum(s);
    }
  }
  if (lane == 0) h.ref[i] = fabsf(best) < INFINITY ? best : 0.f;
}

// The entries of 128 compact rows sorted by groups of 64 columns, for the first product to pick their logits from its accumulators (HeadEpi's offs and list).  The order within a group
// does not matter: every entry has a place of its own for its logit.  A block per 128 rows; dynamic shared memory: `groups` counters.
__global__ __launch_bounds__(1024) void head_lists_kernel(const int32_t* __restrict__ rows, const int32_t* __restrict__ count, const int32_t* __restrict__ ids, const float* __restrict__ logits,
                                                          const unsigned char* __restrict__ flags, int V, int top, int i0, int piece, int groups, int32_t* __restrict__ offs, int32_t* __restrict__ list) {
  extern __shared__ int cnt[];
  __shared__ int wave_sum_s[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, live = min(max(*count - i0, 0), piece), r0 = blockIdx.x * 128;
  for (int g = tid; g < groups; g += 1024) cnt[g] = 0;
  __syncthreads();
  auto each = [&](auto f) {          // f(row in the 128, entry, id)
    for (int x = tid; x < 128 * top; x += 1024) {
      const int r = x / top, j = x - r * top;
      if (r0 + r >= live) break;
      const int t = rows[i0 + r0 + r];
      if (!(flags[t] & ROW_SOFT)) continue;
      const int id = ids[(size_t)t * top + j];
      if ((uint32_t)id < (uint32_t)V && logits[(size_t)t * top + j] != -INFINITY) f(r, j, id);
    }
  };
  each([&](int, int, int id) { atomicAdd(&cnt[id >> 6], 1); });
  __syncthreads();
  // counters to starts, 1024 groups at a time
  int32_t* o = offs + (size_t)blockIdx.x * (groups + 1);
  int base = 0;
  for (int g0 = 0; g0 < groups; g0 += 1024) {
    const int g = g0 + tid, mine = g < groups ? cnt[g] : 0;
    int incl = mine;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const int v = __shfl_up(incl, k, 64);
      if (lane >= k) incl += v;
    }
    __syncthreads();
    if (lane == 63) wave_sum_s[wave] = incl;
    __syncthreads();
    int before = base, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) { const int v = wave_sum_s[w]; if (w < wave) before += v; all += v; }
    if (g < groups) { o[g] = before + incl - mine; cnt[g] = before + incl - mine; }
    base += all;
  }
  if (tid == 0) o[groups] = base;
  __syncthreads();
  int32_t* l = list + (size_t)blockIdx.x * 128 * top;
  each([&](int r, int j, int id) { l[atomicAdd(&cnt[id >> 6], 1)] = r | (id & 63) << 7 | j << 13; });
}

// A block per 16 compact rows of the piece: sums over the column groups in a fixed order, then a wave per row: loss, log-sum-exp, scale g C, and the new values of e at the target and the
// entries.  `again`: only rows of blocks that were done again.
struct HeadFin {
  const float2* stats;
  const float* stats2;          // mixed: sums of the second softmax
  int groups, piece, i0, V, vp, top, mixed, again;
  const int32_t *rows, *count, *targets, *ids;
  const float *logits, *weight, *zsel;
  const unsigned char* flags;
  float *ref, *scale, *row_loss, *row_lse;
  float2* coef;                 // mixed: shares of the two exponentials in e, for head_mix_kernel
  bf16_t* e;                    // nullptr: losses alone
  int places;                   // 1: the places are written
  int32_t* redo;
  float tau, share, k, kt;          // k, kt: HeadEpi's
};
constexpr float kFar = 40.f;          // e <= exp(40): sums of 2^20 of them, times what dX's product adds up, stay far from overflow, and C far from underflow
template <bool OWN>          // sums against the groups' own largest logits
__global__ __launch_bounds__(1024) void head_fin_kernel(HeadFin h) {
  __shared__ float s1_s[64][17], s2_s[64][17], top_s[64][17];          // 17: columns on different banks
  __shared__ __align__(16) int id_s[16][kTopMax];
  __shared__ float q_s[16][kTopMax];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b0 = blockIdx.x * 16, live = min(max(*h.count - h.i0, 0), h.piece);
  if (h.again) { if (!h.redo[0] || !h.redo[1 + b0 / 256]) return; }
  if (b0 >= live) return;
  {
    const int row = min(b0 + (tid & 15), live - 1), slice = tid >> 4;
    float s1 = 0.f, s2 = 0.f, far = -INFINITY;
    const float2* sp = h.stats + row;
    const float* sp2 = h.stats2 + row;
    int g = slice;
    for (; OWN && g < h.groups; g += 64) {          // each group's sum to the largest logit so far
      const float2 v = sp[(size_t)g * h.piece];
      const float u = h.mixed ? sp2[(size_t)g * h.piece] : 0.f, m = fmaxf(far, v.y);
      if (m == -INFINITY) { s1 += v.x; s2 += u; continue; }          // nothing, or NaN
      s1 = s1 * __builtin_amdgcn_exp2f((far - m) * h.k) + v.x * __builtin_amdgcn_exp2f((v.y - m) * h.k);
      s2 = s2 * __builtin_amdgcn_exp2f((far - m) * h.kt) + u * __builtin_amdgcn_exp2f((v.y - m) * h.kt);
      far = m;
    }
    for (; g + 7 * 64 < h.groups; g += 8 * 64) {          // eight loads in flight
      float2 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = sp[(size_t)(g + 64 * k) * h.piece];
#pragma unroll
      for (int k = 0; k < 8; ++k) { s1 += v[k].x; far = fmaxf(far, v[k].y); }
      if (h.mixed) {
        float u[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = sp2[(size_t)(g + 64 * k) * h.piece];
#pragma unroll
        for (int k = 0; k < 8; ++k) s2 += u[k];
      }
    }
    for (; g < h.groups; g += 64) {
      const float2 v = sp[(size_t)g * h.piece];
      s1 += v.x;
      far = fmaxf(far, v.y);
      if (h.mixed) s2 += sp2[(size_t)g * h.piece];
    }
    s1_s[slice][tid & 15] = s1; s2_s[slice][tid & 15] = s2; top_s[slice][tid & 15] = far;
  }
  __syncthreads();
  if (b0 + wave >= live) return;
  {
    const int r = wave;          // a row per wave from here on
    const float far = wave_max(top_s[lane][r]);
    float sl = s1_s[lane][r], sl2 = s2_s[lane][r];
    if (OWN && far != -INFINITY) {
      sl *= __builtin_amdgcn_exp2f((top_s[lane][r] - far) * h.k);
      sl2 *= __builtin_amdgcn_exp2f((top_s[lane][r] - far) * h.kt);
    }
    const float sa = wave_sum(sl), st = h.mixed ? wave_sum(sl2) : sa;          // of the hard targets' softmax and of the teacher's (one and the same unless mixed)
    // Largest exponent, of the sharper one of two softmaxes, as a power of two.  Such a row takes its maximum as reference (what the rest of this
    // kernel makes of it is overwritten when its block is done again).  Below -kFar: the reference was 0, those logits not being finite.  A row of a weight below 2^-40 has no room for a
    // sum of exp(40) in its scale: it takes its maximum too.
    const int i = h.i0 + b0 + r, t = h.rows[i];
    const float weight = h.weight ? h.weight[t] : 1.0f / (float)*h.count;
    const float span = far * 0.693147181f, most_span = h.e && fabsf(weight) < 0x1p-40f ? 1.f : kFar;
    if (!OWN && !h.again && fabsf(span) > most_span && fabsf(far) < 1e30f && lane == 0) {
      h.ref[i] += span * (h.mixed ? fminf(1.f, h.tau) : h.tau);
      h.redo[0] = 1;
      h.redo[1 + b0 / 256] = 1;
    }
    const bool hard = h.flags ? h.flags[t] & ROW_HARD : true, soft = h.flags ? h.flags[t] & ROW_SOFT : false;
    const float ref = OWN ? (far == -INFINITY ? 0.f : far) : h.ref[i], it = 1.0f / h.tau;
    const float* zs = h.zsel + (size_t)i * (h.top + 1);
    const int y = hard ? h.targets[t] : -1;
    const float zy = hard ? zs[h.top] : 0.f;
    // the teacher's softmax over its entries, two per lane
    int id[2] = {-1, -1};
    float q[2] = {0.f, 0.f}, zj[2] = {0.f, 0.f};
    float l = 0.f;
    if (soft) {
      float u[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int j = lane + 64 * k;
        if (j < h.top) {
          id[k] = h.ids[(size_t)t * h.top + j];
          if ((uint32_t)id[k] < (uint32_t)h.V) u[k] = h.logits[(size_t)t * h.top + j]; else id[k] = -1;
          if (u[k] == -INFINITY) id[k] = -1;
          if (id[k] >= 0) zj[k] = zs[j];
        }
      }
      const float m = wave_max(fmaxf(id[0] >= 0 ? u[0] : -INFINITY, id[1] >= 0 ? u[1] : -INFINITY));
#pragma unroll
      for (int k = 0; k < 2; ++k) q[k] = id[k] >= 0 ? expf((u[k] - m) * it) : 0.f;
      const float sum = wave_sum(q[0] + q[1]), lst = logf(st);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        q[k] /= sum;
        if (id[k] >= 0 && !(q[k] <= 0.f)) l += q[k] * (logf(q[k]) - (zj[k] - ref) * it + lst);
      }
      l = wave_sum(l) * h.share * h.tau * h.tau;
    }
    if (hard) l += (1.f - h.share) * ((ref - zy) + logf(sa));
    if (lane == 0) {
      h.row_loss[t] = l;
      if (h.row_lse) h.row_lse[t] = ref * it + logf(st);
    }
    if (!h.e) return;
    // dz = g (p1 e1 + pt et - sub).  The larger coefficient goes into g: 1 / C stays finite whatever the row's weight and share, and g is in the row's scale alone.
    const float k1 = hard ? 1.f - h.share : 0.f, kt = soft ? h.share * h.tau : 0.f, most = fmaxf(fmaxf(k1, kt), 1e-37f);
    const float g = weight * most, c1 = k1 / most, ct = kt / most;
    const float p1 = c1 / sa, pt = ct / st, C = p1 + pt;
    const float inv = C != 0.f ? 1.0f / C : 0.f;
    if (h.coef && lane == 0) h.coef[b0 + r] = make_float2(p1 * inv, pt * inv);
    if (!h.places) return;
    // e at the places, in fp32: the softmaxes' part from the place's logit, less what is taken off there.  The first of equal ids stands for all, in their order; lane 0
    // holds the target in its third slot unless it is among the entries.
#pragma unroll
    for (int k = 0; k < 2; ++k)
      { id_s[wave][lane + 64 * k] = id[k]; q_s[wave][lane + 64 * k] = q[k]; }          // -1 behind the last entry
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): this wave's own list
    auto place = [&](float zv, float sub) {
      const float e1 = p1 != 0.f ? p1 * expf((zv - ref) * (h.mixed ? 1.f : it)) : 0.f, et = pt != 0.f ? pt * expf((zv - ref) * it) : 0.f;
      return (e1 + et - sub) * inv;
    };
    int at[3] = {-1, -1, -1};
    float val[3] = {0.f, 0.f, 0.f};
    bool y_listed = false;
    int same[2] = {0, 0};          // entries with this id
    if (soft) {
#pragma unroll 4
      for (int o = 0; o < h.top; o += 4) {
        const int4 v = *reinterpret_cast<const int4*>(&id_s[wave][o]);
#pragma unroll
        for (int k = 0; k < 2; ++k) same[k] += (v.x == id[k]) + (v.y == id[k]) + (v.z == id[k]) + (v.w == id[k]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int j = lane + 64 * k;
        if (j < h.top && id[k] >= 0) {
          y_listed |= id[k] == y;
          bool first = true;
          float sub = ct * q[k];
          if (same[k] > 1) {
            sub = 0.f;
            for (int o = 0; o < h.top; ++o)
              if (id_s[wave][o] == id[k]) { if (o < j) first = false; sub += ct * q_s[wave][o]; }
          }
          if (first) { at[k] = id[k]; val[k] = place(zj[k], id[k] == y ? sub + c1 : sub); }
        }
      }
    }
    if (hard && !__ballot(y_listed) && lane == 0) { at[2] = y; val[2] = place(zy, c1); }
    // The row of dz is g C e.  Most of its length lies in the largest place (at the target p - 1 against many small p), so C is moved by the at most 2^-8 that make that place's rounded
    // value exact: the error that is left is that of the row's smaller part, where the move is of the size of the other elements' own rounding (1024 x 768 x 32000, target first: dX 1.66e-3 from the
    // exact values in place of 2.35e-3, 1.66e-3 of it the result's own rounding; dW 1.86e-3 in place of 2.05e-3; a row's sum is as far from 0 with it as without, 1.3e-3 of its weight).
    float big = fmaxf(fmaxf(fabsf(val[0]), fabsf(val[1])), fabsf(val[2]));
    big = wave_max(big);
    const float rounded = bf16_to_f32(f32_to_bf16(big));
    const float move = big > 0.f && big < 1e37f ? rounded / big : 1.f;          // exact e -> stored e
    if (lane == 0) h.scale[i] = g * (C / move);
    bf16_t* e = h.e + (size_t)(b0 + r) * h.vp;
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (at[k] >= 0) e[at[k]] = from_f32<bf16_t>(val[k] * move);
  }
}

// Two softmaxes: the stored exponents (head_exponent_code) become (p1 e1 + pt et) / C, in front of head_fin's places.  k1, kt: of the two softmaxes in units of the sharper one's exponent,
// which is the one that is stored.  A block per row and 8192 columns.
__global__ __launch_bounds__(256) void head_mix_kernel(bf16_t* e, int vp, const float2* __restrict__ coef, const int32_t* __restrict__ count, int i0, int piece, float k1, float kt) {
  const int i = blockIdx.x, v0 = blockIdx.y * 1024 + threadIdx.x;
  if (i >= min(max(*count - i0, 0), piece)) return;
  const float2 c = coef[i];
  uint4* row = reinterpret_cast<uint4*>(e + (size_t)i * vp);
  uint4 r[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) r[m] = row[min(v0 + 256 * m, vp / 8 - 1)];
  auto mixed = [&](uint32_t code) {
    const float y = head_exponent(code);
    return c.x * __builtin_amdgcn_exp2f(y * k1) + c.y * __builtin_amdgcn_exp2f(y * kt);
  };
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    uint32_t w[4] = {r[m].x, r[m].y, r[m].z, r[m].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = f32x2_to_bf16x2(mixed(w[k] & 0xffff), mixed(w[k] >> 16));
    if (v0 + 256 * m < vp / 8) row[v0 + 256 * m] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// dst[c][i] = scale[i] x[i][c] for the compact rows of a piece (live64 of them): X's rows as dW's product reads them, rounded to bf16 once more: the scale is
// known only after the exponentials are stored, and as a factor of X it costs no pass over them (dW 1.66e-3 -> 1.86e-3 from the exact values over 1024 rows, 1.64e-3 -> 2.1e-3 where 395 rows have weights of their own)
__global__ __launch_bounds__(256) void head_xt_kernel(const bf16_t* __restrict__ x, int dp, const float* __restrict__ scale, bf16_t* __restrict__ dst, int ld_dst, int d, const int32_t* __restrict__ count,
                                                      int i0, int piece) {
  __shared__ uint16_t tile[64][72];
  const int live = min(max(*count - i0, 0), piece), r0 = blockIdx.x * 64, c0 = blockIdx.y * 64, t = threadIdx.x;
  if (r0 >= live) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (t >> 3) + 32 * i, c8 = (t & 7) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (r0 + r < live) {
      load8(x + (size_t)(r0 + r) * dp + c0 + c8, v);
      const float s = scale[i0 + r0 + r];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= s;
    }
    store8(reinterpret_cast<bf16_t*>(&tile[r][c8]), v);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = (t >> 3) + 32 * i, r8 = (t & 7) * 8;
    if (c0 + c >= d) continue;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = (uint32_t)tile[r8 + 2 * k][c] | ((uint32_t)tile[r8 + 2 * k + 1][c] << 16);
    *reinterpret_cast<uint4*>(dst + (size_t)(c0 + c) * ld_dst + r0 + r8) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// ------------------------------------------------------------------------------------------------ few rows
// Up to 16 rows (one block of a 16 x 16 MFMA, whichever storage type): W is streamed once for the losses, by waves that take 16 of its rows at a time from memory straight into
// MFMA operands, and once for dX; dW is written once.  Bound by those bytes: 32000 x 2048 bf16 (131 MB) at the card's copy rate 25 us.  Logits in fp32 (16 rows of them at most),
// dz in fp32 and not rounded.  Fixed orders throughout: no atomics.
struct HeadFew {
  const void *x, *w;
  int ldx, ldw, n, V, d, ldz, parts, top, dw_lo, dw_hi, lddx, lddw, dw_add, chunk, chunk_dw;          // parts: waves of the first kernel; chunk, chunk_dw: rows of W per workgroup of dX's and dW's
  const int32_t *targets, *ids;
  const float *logits, *weight;
  float tau, share;
  float *z, *part, *coef, *sub, *psum;          // z [n][ldz], part [16][parts / 4][4], coef [16][4], sub [16][top + 1], psum [partials][n][d]
  int32_t *sid;                                 // [16][top + 1]: where sub is taken off, -1: nowhere
  float *loss, *row_loss, *row_lse;
  void *dx, *dw;
};
typedef float few_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 few_bf16x8 __attribute__((ext_vector_type(8)));
template <class T> struct FewChunk;          // 16 bytes of a row: 8 bf16 or 4 floats
template <> struct FewChunk<bf16_t> { static constexpr int E = 8; };
template <> struct FewChunk<float> { static constexpr int E = 4; };

template <class T> __device__ __forceinline__ uint4 few_load(const T* row, int k, int d) {          // elements k .. of a row, zeros from d on
  constexpr int E = FewChunk<T>::E;
  if (k + E <= d) {
    const any16 r = *reinterpret_cast<const any16*>(row + k);
    return make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
  }
  if (k >= d) return make_uint4(0, 0, 0, 0);
  union { uint4 u; T e[E]; } r;
#pragma unroll
  for (int i = 0; i < E; ++i) r.e[i] = k + i < d ? row[k + i] : from_f32<T>(0.f);
  return r.u;
}
__device__ __forceinline__ void few_load8(const bf16_t* p, float v[8]) {
  const any16 r = *reinterpret_cast<const any16*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r.w[i] << 16); v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void few_load8(const float* p, float v[8]) {
  const any16 a = *reinterpret_cast<const any16*>(p), b = *reinterpret_cast<const any16*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a.w[i]); v[4 + i] = __uint_as_float(b.w[i]); }
}
__device__ __forceinline__ void few_mfma(few_f32x4& acc, const uint4& a, const uint4& b, bf16_t) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(few_bf16x8, a), __builtin_bit_cast(few_bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void few_mfma(few_f32x4& acc, const uint4& a, const uint4& b, float) {          // the four k of a lane's chunk, one per MFMA
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
}
// (m, s) of a softmax's maximum and sum, s2 the sum at the teacher's temperature
__device__ __forceinline__ void few_merge(float& m, float& s, float& s2, float mo, float so, float so2, float it) {
  const float top = fmaxf(m, mo);
  if (top == -INFINITY) { s += so; s2 += so2; return; }          // nothing yet on either side (or only NaN, which both keep)
  const float a = expf(m - top), b = expf(mo - top);
  s = s * a + so * b;
  s2 = it == 1.f ? s : s2 * expf((m - top) * it) + so2 * expf((mo - top) * it);
  m = top;
}

template <class T, bool SPLIT>          // SPLIT: a quarter of 16 rows of W for each of a workgroup's waves
__global__ __launch_bounds__(256) void head_few_z_kernel(HeadFew h) {
  constexpr int E = FewChunk<T>::E, U = 8, STEP = 4 * E;          // k per MFMA step of the four lane groups
  const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4, gw = blockIdx.x * 4 + (threadIdx.x >> 6);
  const T* x = (const T*)h.x + (size_t)min(l16, h.n - 1) * h.ldx;
  const float it = 1.0f / h.tau;
  float m = -INFINITY, s = 0.f, s2 = 0.f;
  [[maybe_unused]] __shared__ few_f32x4 acc_s[4][64];
  const int wave = threadIdx.x >> 6, quarter = SPLIT ? (h.d + 4 * STEP - 1) / (4 * STEP) * STEP : h.d;
  const int kb = SPLIT ? wave * quarter : 0, ke = min(kb + quarter, h.d);
  for (int tile = SPLIT ? blockIdx.x : gw; tile * 16 < h.V; tile += SPLIT ? gridDim.x : h.parts) {
    const T* w = (const T*)h.w + (size_t)min(tile * 16 + l16, h.V - 1) * h.ldw;
    few_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    uint4 a[2][U], b[2][U];
    auto fetch = [&](int buf, int k0) {
#pragma unroll
      for (int u = 0; u < U; ++u) a[buf][u] = few_load<T>(w, k0 + u * STEP + lq * E, ke);
#pragma unroll
      for (int u = 0; u < U; ++u) b[buf][u] = few_load<T>(x, k0 + u * STEP + lq * E, ke);
    };
    auto multiply = [&](int buf) {
#pragma unroll
      for (int u = 0; u < U; ++u) few_mfma(acc, a[buf][u], b[buf][u], T{});
    };
    fetch(0, kb);
    for (int k0 = kb; k0 < ke; k0 += 2 * U * STEP) {          // chunks behind the last are zeros without a load
      fetch(1, k0 + U * STEP);
      multiply(0);
      fetch(0, k0 + 2 * U * STEP);
      multiply(1);
    }
    if constexpr (SPLIT) {          // the quarters in their order; the first wave goes on with the sum
      acc_s[wave][lane] = acc;
      __syncthreads();
      acc = acc_s[0][lane] + acc_s[1][lane] + acc_s[2][lane] + acc_s[3][lane];
      __syncthreads();
      if (wave) continue;
    }
    // element r: row 4 lq + r of the 16 rows of W, token l16
    const int v0 = tile * 16 + 4 * lq;
    if (l16 < h.n) *reinterpret_cast<float4*>(h.z + (size_t)l16 * h.ldz + v0) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    float tm = -INFINITY, ts = 0.f, ts2 = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (v0 + r >= h.V) acc[r] = -INFINITY;
      tm = fmaxf(tm, acc[r]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (acc[r] != -INFINITY) { ts += expf(acc[r] - tm); if (it != 1.f) ts2 += expf((acc[r] - tm) * it); }
    few_merge(m, s, s2, tm, ts, it == 1.f ? ts : ts2, it);
  }
#pragma unroll
  for (int o = 16; o < 64; o <<= 1) few_merge(m, s, s2, __shfl_xor(m, o, 64), __shfl_xor(s, o, 64), __shfl_xor(s2, o, 64), it);
  // the workgroup's four waves, in their order
  __shared__ float4 sum_s[4][16];
  if (lq == 0) sum_s[threadIdx.x >> 6][l16] = make_float4(m, s, s2, 0.f);
  __syncthreads();
  if (threadIdx.x >= 16) return;
  for (int k = 1; k < 4; ++k) {
    const float4 o = sum_s[k][l16];
    few_merge(m, s, s2, o.x, o.y, o.z, it);
  }
  *reinterpret_cast<float4*>(h.part + ((size_t)l16 * gridDim.x + blockIdx.x) * 4) = make_float4(m, s, s2, 0.f);
}

// One block, a wave per row: losses, and for the gradients dz = coef[1] exp(z - coef[0]) + coef[2] exp((z - coef[0]) / tau) - sub at sid (all 0 for a row that is left out)
__global__ __launch_bounds__(1024) void head_few_fin_kernel(HeadFew h) {
  __shared__ int live_s[kFew], id_s[kFew][kTopMax];
  __shared__ float loss_s[kFew], q_s[kFew][kTopMax];
  const int lane = threadIdx.x & 63, t = threadIdx.x >> 6;
  const float it = 1.0f / h.tau, w = t < h.n && h.weight ? h.weight[t] : 1.f;
  int id[2] = {-1, -1};
  float u[2] = {-INFINITY, -INFINITY}, q[2] = {0.f, 0.f};
  bool hard = false, soft = false;
  float l = 0.f, lse = 0.f, m = -INFINITY, s = 0.f, s2 = 0.f;
  if (t < h.n) {
    hard = w != 0.f && hard_row(h.targets, t, h.V);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = lane + 64 * k;
      if (j < h.top && h.share > 0.f && w != 0.f) {
        id[k] = h.ids[(size_t)t * h.top + j];
        if ((uint32_t)id[k] < (uint32_t)h.V) u[k] = h.logits[(size_t)t * h.top + j]; else id[k] = -1;
        if (u[k] == -INFINITY) id[k] = -1;
      }
    }
    soft = __ballot(id[0] >= 0 || id[1] >= 0) != 0;
    // at most 512 partial sums, 8 a lane: all of them requested at once, the maximum first, then sums that do not wait for each other
    const int parts = h.parts / 4;
    const float4* part = reinterpret_cast<const float4*>(h.part) + (size_t)t * parts;
    constexpr int K = 2048 / 4 / 64;
    float4 p[K];
#pragma unroll
    for (int k = 0; k < K; ++k) p[k] = lane + 64 * k < parts ? part[lane + 64 * k] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) m = fmaxf(m, p[k].x);
    m = wave_max(m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      s += p[k].x == -INFINITY ? p[k].y : p[k].y * expf(p[k].x - m);          // a part without a finite logit has a sum of 0, or NaN
      if (it != 1.f) s2 += p[k].x == -INFINITY ? p[k].z : p[k].z * expf((p[k].x - m) * it);
    }
    s = wave_sum(s);
    s2 = it == 1.f ? s : wave_sum(s2);
  }
  if (lane == 0) live_s[t] = hard || soft;
  __syncthreads();
  int count = 0;
  for (int k = 0; k < kFew; ++k) count += live_s[k];
  const bool live = hard || soft;
  const float* z = h.z + (size_t)min(t, h.n - 1) * h.ldz;
  const int y = hard ? h.targets[t] : -1;
  const float zy = hard ? z[y] : 0.f;
  float zj[2] = {0.f, 0.f};
  if (soft) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (id[k] >= 0) zj[k] = z[id[k]];
    const float um = wave_max(fmaxf(id[0] >= 0 ? u[0] : -INFINITY, id[1] >= 0 ? u[1] : -INFINITY));
#pragma unroll
    for (int k = 0; k < 2; ++k) q[k] = id[k] >= 0 ? expf((u[k] - um) * it) : 0.f;
    const float sum = wave_sum(q[0] + q[1]), lst = logf(s2);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      q[k] /= sum;
      if (id[k] >= 0 && !(q[k] <= 0.f)) l += q[k] * (logf(q[k]) - (zj[k] - m) * it + lst);
    }
    l = wave_sum(l) * h.share * h.tau * h.tau;
  }
  if (hard) l += (1.f - h.share) * ((m - zy) + logf(s));
  if (live) lse = m * it + logf(s2);
  const float g = h.weight ? w : 1.0f / (float)max(count, 1);
  if (t < h.n && lane == 0) { h.row_loss[t] = l; if (h.row_lse) h.row_lse[t] = lse; }
  if (lane == 0) loss_s[t] = live ? (h.weight ? w * l : l) : 0.f;
  // gradients' coefficients
  const float c1 = hard ? g * (1.f - h.share) : 0.f, ct = soft ? g * h.share * h.tau : 0.f;
  if (lane == 0) *reinterpret_cast<float4*>(h.coef + t * 4) = make_float4(m, hard ? c1 / s : 0.f, soft ? ct / s2 : 0.f, live ? 1.f : 0.f);
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (lane + 64 * k < h.top) { id_s[t][lane + 64 * k] = id[k]; q_s[t][lane + 64 * k] = q[k]; }
  __syncthreads();
  bool y_listed = false;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 64 * k;
    if (j >= h.top) continue;
    bool first = id[k] >= 0;
    float sub = id[k] == y ? c1 : 0.f;
    y_listed |= hard && id[k] == y;
    if (id[k] >= 0)
      for (int o = 0; o < h.top; ++o)
        if (id_s[t][o] == id[k]) { if (o < j) first = false; sub += ct * q_s[t][o]; }
    h.sid[t * (h.top + 1) + j] = first ? id[k] : -1;
    h.sub[t * (h.top + 1) + j] = sub;
  }
  const bool listed = __ballot(y_listed) != 0;
  if (lane == 0) { h.sid[t * (h.top + 1) + h.top] = hard && !listed ? y : -1; h.sub[t * (h.top + 1) + h.top] = c1; }
  if (threadIdx.x == 0 && h.loss) {
    float a = 0.f;
    for (int k = 0; k < kFew; ++k) a += loss_s[k];
    *h.loss = h.weight ? a : a / (float)max(count, 1);
  }
}

// dz[r][t] of rows v0 .. v0 + rows - 1 of W for NT tokens into shared memory; every thread calls it
template <int NT>
__device__ __forceinline__ void few_dz(const HeadFew& h, int v0, int rows, float (*dz)[NT]) {
  const float it = 1.0f / h.tau;
  __syncthreads();
  const int lg = 32 - __clz(max(rows - 1, 1)), all = NT << lg;          // 2 ^ lg >= rows
  constexpr int K = NT < 8 ? 1 : NT / 4;          // elements of a thread at a time, their loads in flight together
  for (int i0 = threadIdx.x; i0 < all; i0 += 256 * K) {
    float4 c[K];
    float z[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = i0 + 256 * k, t = min(i >> lg, h.n - 1), r = min(i & ((1 << lg) - 1), rows - 1);
      c[k] = *reinterpret_cast<const float4*>(h.coef + t * 4);
      z[k] = h.z[(size_t)t * h.ldz + v0 + r];
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = i0 + 256 * k, t = i >> lg, r = i & ((1 << lg) - 1);
      if (i >= all) break;
      const float a = z[k] - c[k].x;
      dz[r][t] = t < h.n && r < rows && c[k].w != 0.f ? (c[k].y != 0.f ? c[k].y * expf(a) : 0.f) + (c[k].z != 0.f ? c[k].z * expf(a * it) : 0.f) : 0.f;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < h.n * (h.top + 1); i += 256) {          // no two entries of a row have the same place
    const int t = i / (h.top + 1), v = h.sid[i];
    if (v >= v0 && v < v0 + rows) dz[v - v0][t] -= h.sub[i];
  }
  __syncthreads();
}
// Threads of a workgroup: `cols` of them side by side, 8 columns each, 256 / cols rows of W at a time
template <class T>
__device__ __forceinline__ void few_dx(const HeadFew& h, int cols, float (*dz)[1], float* red) {          // one row of X
  const int rp = 256 / cols, cg = threadIdx.x % cols, rg = threadIdx.x / cols, c = (blockIdx.y * cols + cg) * 8;
  const int lo = blockIdx.x * h.chunk, hi = min(lo + h.chunk, h.V);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  const T* w = (const T*)h.w;
  for (int v0 = lo; v0 < hi; v0 += 128) {
    const int rows = min(128, hi - v0);
    few_dz<1>(h, v0, rows, dz);
    if (c >= h.d) continue;          // uniform barriers: few_dz is reached by every thread at every trip
    auto row = [&](int r) {
      float v[8];
      const T* p = w + (size_t)(v0 + r) * h.ldw + c;
      if (c + 8 <= h.d) few_load8(p, v);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < h.d ? to_f32(p[e]) : 0.f;
      const float g = dz[r][0];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(g, v[e], acc[e]);
    };
    int r = rg;
    for (; r + 3 * rp < rows; r += 4 * rp) { row(r); row(r + rp); row(r + 2 * rp); row(r + 3 * rp); }
    for (; r < rows; r += rp) row(r);
  }
  // The workgroup's sums of a column: lanes of a wave, then waves one after the other by way of shared memory, the last one stores
  for (int o = cols; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
  const int rows_at = cols <= 64 ? threadIdx.x >> 6 : rg, last = cols <= 64 ? 3 : rp - 1;
  const bool holds = cols >= 64 || (threadIdx.x & 63) < cols;
  float* out = h.psum + (size_t)blockIdx.x * h.d;
  for (int k = 0; k <= last; ++k) {
    if (rows_at == k && holds) {
      float* at = red + ((cg * 8) & 1023);          // cols 256: one row at a time, nothing to add
      if (k > 0)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += at[e];
      if (k < last)
#pragma unroll
        for (int e = 0; e < 8; ++e) at[e] = acc[e];
      else
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < h.d) out[c + e] = acc[e];
    }
    __syncthreads();
  }
}
// dx = sum of the partials, a block per row and 64 columns, 16 waves of partials
template <class T>
__global__ __launch_bounds__(1024) void head_few_sum_kernel(HeadFew h, int partials) {
  __shared__ float s_s[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = blockIdx.y, c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < h.d)
    for (int p = wave; p < partials; p += 8 * 16) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p + 16 * k < partials ? h.psum[((size_t)(p + 16 * k) * h.n + t) * h.d + c] : 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
  s_s[wave][lane] = s;
  __syncthreads();
  if (wave || c >= h.d) return;
  for (int k = 1; k < 16; ++k) s += s_s[k][lane];
  ((T*)h.dx)[(size_t)t * h.lddx + c] = from_f32<T>(h.coef[t * 4 + 3] != 0.f ? s : 0.f);
}
template <class T, class TO>
__device__ __forceinline__ void few_dw(const HeadFew& h, int cols, int group, float (*dz)[1]) {          // one row of X
  const int rp = 256 / cols, cg = threadIdx.x % cols, rg = threadIdx.x / cols, c = (blockIdx.y * cols + cg) * 8;
  const int lo = h.dw_lo + group * h.chunk_dw, hi = min(lo + h.chunk_dw, h.dw_hi);
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = c + e < h.d && h.coef[3] != 0.f ? to_f32(((const T*)h.x)[c + e]) : 0.f;
  for (int v0 = lo; v0 < hi; v0 += 128) {
    const int rows = min(128, hi - v0);
    few_dz<1>(h, v0, rows, dz);
    if (c >= h.d) continue;
    for (int r = rg; r < rows; r += rp) {
      const float g = dz[r][0];
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = g * x[e];
      TO* p = (TO*)h.dw + (size_t)(v0 + r - h.dw_lo) * h.lddw + c;
      const bool whole = c + 8 <= h.d && h.lddw % 8 == 0 && ((uintptr_t)h.dw & 15) == 0;
      if (h.dw_add)
#pragma unroll
        for (int e = 0; e < 8; ++e) if (c + e < h.d) o[e] += to_f32(p[e]);
      if (whole) store8(p, o);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) if (c + e < h.d) p[e] = from_f32<TO>(o[e]);
    }
  }
}

// dX of several rows by fp32 MFMAs: four rows of W at a time are the second operand, a lane's eight columns eight instructions apart, dz of those rows the first.  16 tokens cost the vector units
// 128 multiply-adds for 16 bytes of W, more than the memory takes to deliver them (dX and dW of 16 x 768 x 32000 115 -> 77 us, 8 x 512 x 5000 47 -> 23).
template <class T, int NT>
__device__ __forceinline__ void few_dx_mfma(const HeadFew& h, int waves, float (*dz)[NT], float (*red)[256]) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4, wave = threadIdx.x >> 6;
  const int wcol = wave % waves, wrow = wave / waves, rows_at = 4 * (4 / waves), c0 = (blockIdx.y * waves + wcol) * 128, c = c0 + l16 * 8;
  const int lo = blockIdx.x * h.chunk, hi = min(lo + h.chunk, h.V);
  few_f32x4 acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = few_f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
  for (int v0 = lo; v0 < hi; v0 += 128) {
    const int rows = min(128, hi - v0);
    few_dz<NT>(h, v0, rows, dz);
    if (c0 >= h.d) continue;          // uniform barriers: few_dz is reached by every thread at every trip
    for (int r = 4 * wrow; r < rows; r += U * rows_at) {
      float w[U][8], a[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int rr = r + u * rows_at + lq;
        const T* p = (const T*)h.w + (size_t)(v0 + min(rr, rows - 1)) * h.ldw + c;
        if (c + 8 <= h.d) few_load8(p, w[u]);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) w[u][e] = c + e < h.d ? to_f32(p[e]) : 0.f;
        a[u] = rr < rows && l16 < NT ? dz[rr][l16 & (NT - 1)] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u], w[u][e], acc[e], 0, 0, 0);
    }
  }
  // element r of acc[e]: token 4 lq + r, column c + e.  Waves of the same columns one after the other by way of shared memory, the last one stores.
  float* out = h.psum + (size_t)blockIdx.x * h.n * h.d;
  const int last = 4 / waves - 1;
  for (int k = 0; k <= last; ++k) {
    if (wrow == k)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float* at = &red[4 * lq + r][(wcol * 128 + l16 * 8) & 255];          // four waves side by side: nothing to add
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = acc[e][r] + (k > 0 ? at[e] : 0.f);
        if (k < last) {
#pragma unroll
          for (int e = 0; e < 8; ++e) at[e] = v[e];
        } else if (4 * lq + r < h.n) {
          float* o = out + (size_t)(4 * lq + r) * h.d;
          store_cols(o, c, h.d, make_float4(v[0], v[1], v[2], v[3]));
          store_cols(o, c + 4, h.d, make_float4(v[4], v[5], v[6], v[7]));
        }
      }
    __syncthreads();
  }
}

// dW of several rows likewise: 16 rows of W at a time, dz of four tokens the first operand, their rows of X (held by the lanes) the second
template <class T, class TO, int NT>
__device__ __forceinline__ void few_dw_mfma(const HeadFew& h, int waves, int group, float (*dz)[NT]) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4, wave = threadIdx.x >> 6;
  const int wcol = wave % waves, wrow = wave / waves, c0 = (blockIdx.y * waves + wcol) * 128, c = c0 + l16 * 8;
  const int lo = h.dw_lo + group * h.chunk_dw, hi = min(lo + h.chunk_dw, h.dw_hi);
  float x[NT / 4][8];
#pragma unroll
  for (int s = 0; s < NT / 4; ++s) {
    const int t = 4 * s + lq;
    const bool there = t < h.n && h.coef[t * 4 + 3] != 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[s][e] = there && c + e < h.d ? to_f32(((const T*)h.x)[(size_t)t * h.ldx + c + e]) : 0.f;
  }
  for (int v0 = lo; v0 < hi; v0 += 128) {
    const int rows = min(128, hi - v0);
    few_dz<NT>(h, v0, rows, dz);
    if (c0 >= h.d) continue;
    for (int r0 = 16 * wrow; r0 < rows; r0 += 16 * (4 / waves)) {
      few_f32x4 acc[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = few_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NT / 4; ++s) {
        const float a = r0 + l16 < rows ? dz[r0 + l16][4 * s + lq] : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, x[s][e], acc[e], 0, 0, 0);
      }
      // element r of acc[e]: row 4 lq + r, column c + e
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = r0 + 4 * lq + r;
        if (row >= rows) continue;
        TO* p = (TO*)h.dw + (size_t)(v0 + row - h.dw_lo) * h.lddw;
        float4 o0 = make_float4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]), o1 = make_float4(acc[4][r], acc[5][r], acc[6][r], acc[7][r]);
        if constexpr (sizeof(TO) == 4)
          if (h.dw_add) {
            const float4 b0 = load_cols((const float*)p, c, h.d), b1 = load_cols((const float*)p, c + 4, h.d);
            o0.x += b0.x; o0.y += b0.y; o0.z += b0.z; o0.w += b0.w;
            o1.x += b1.x; o1.y += b1.y; o1.z += b1.z; o1.w += b1.w;
          }
        if (sizeof(TO) == 2 && c + 8 <= h.d)
          *reinterpret_cast<any16*>(p + c) = any16{{f32x2_to_bf16x2(o0.x, o0.y), f32x2_to_bf16x2(o0.z, o0.w), f32x2_to_bf16x2(o1.x, o1.y), f32x2_to_bf16x2(o1.z, o1.w)}};
        else {
          store_cols(p, c, h.d, o0);
          store_cols(p, c + 4, h.d, o1);
        }
      }
    }
  }
}

// The first `groups` workgroups form dX's partial sums, the others dW: neither waits for the other, so they share a launch (8 x 512 x 5000 60.6 -> 55.4 us, one row of 2048 x 32000 90 -> 81)
template <class T, class TO, int NT>
__global__ __launch_bounds__(256) void head_few_grads_kernel(HeadFew h, int cols, int waves, int groups) {
  __shared__ __align__(16) float dz[128][NT];
  __shared__ float red[NT == 1 ? 1024 : 16 * 256];
  if ((int)blockIdx.x < groups) {
    if constexpr (NT == 1) few_dx<T>(h, cols, dz, red);
    else few_dx_mfma<T, NT>(h, waves, dz, reinterpret_cast<float(*)[256]>(red));
  } else if constexpr (NT == 1)
    few_dw<T, TO>(h, cols, blockIdx.x - groups, dz);
  else
    few_dw_mfma<T, TO, NT>(h, waves, blockIdx.x - groups, dz);
}

// ------------------------------------------------------------------------------------------------ outputs
// Sum of the partials [splits][pitch] at one place of four columns, in their order, eight loads in flight
__device__ __forceinline__ float4 sum_partials(const float* part, int splits, size_t pitch, int c, int d) {
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int z = 0; z < splits; z += 8) {
    float4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = z + k < splits ? load_cols(part + (z + k) * pitch, c, d) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 8; ++k) { s.x += v[k].x; s.y += v[k].y; s.z += v[k].z; s.w += v[k].w; }
  }
  return s;
}
// A row takes as many lanes of a wave as it has groups of four columns, 1 << lg, and up to 64: narrow rows share a wave.
static int row_lanes(int d) { int lg = 0; while (lg < 6 && (4 << lg) < d) ++lg; return lg; }
static dim3 row_grid(int rows, int d) { const int per = 256 >> row_lanes(d); return dim3((rows + per - 1) / per, (d + 255) / 256); }
// dx[rows[i]] = scale[i] (1 without) sum of the partials [splits][pitch][d] for the compact rows of the piece; pitch 0: the rows that count, in whole groups of 64
template <class T>
__global__ __launch_bounds__(256) void head_dx_sum_kernel(const float* __restrict__ part, int splits, const int32_t* __restrict__ splits_dev, int pitch, const float* __restrict__ scale, T* __restrict__ dx, int lddx, int d,
                                                          const int32_t* __restrict__ rows, const int32_t* __restrict__ count, int i0, int piece, int lg) {
  const int i = blockIdx.x * (256 >> lg) + (threadIdx.x >> lg), live = min(max(*count - i0, 0), piece), c = blockIdx.y * 256 + (threadIdx.x & ((1 << lg) - 1)) * 4;
  if (i >= live || c >= d) return;
  if (splits_dev) { splits = *splits_dev; if (splits == 1) return; }          // then the product's own kernel wrote dx
  const float sc = scale ? scale[i0 + i] : 1.f;
  const int t = rows[i0 + i];
  float4 s = sum_partials(part + (size_t)i * d, splits, (size_t)(pitch ? pitch : (live + 63) & ~63) * d, c, d);
  s.x *= sc; s.y *= sc; s.z *= sc; s.w *= sc;
  store_cols(dx + (size_t)t * lddx, c, d, s);
}
// out = sum of the partials [splits][rows][d] (+ add), out float or bf16
template <class TO>
__global__ __launch_bounds__(256) void head_dw_sum_kernel(const float* __restrict__ part, int splits, const float* add, int ldadd, TO* out, int ldo, int rows, int d, int lg) {
  const int r = blockIdx.x * (256 >> lg) + (threadIdx.x >> lg), c = blockIdx.y * 256 + (threadIdx.x & ((1 << lg) - 1)) * 4;
  if (r >= rows || c >= d) return;
  float4 s = sum_partials(part + (size_t)r * d, splits, (size_t)rows * d, c, d);
  if (add) {
    const float4 a = load_cols(add + (size_t)r * ldadd, c, d);
    s.x += a.x; s.y += a.y; s.z += a.z; s.w += a.w;
  }
  store_cols(out + (size_t)r * ldo, c, d, s);
}
template <class TO>
__global__ __launch_bounds__(256) void head_zero_kernel(TO* out, int ldo, int rows, int d) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  for (int c = threadIdx.x & 63; c < d; c += 64) out[(size_t)r * ldo + c] = from_f32<TO>(0.f);
}
// loss = sum of weight * row_loss, or their mean over the rows that count (rows that are left out have a row_loss of 0, and their weight is not looked at)
__global__ __launch_bounds__(1024) void head_loss_kernel(const float* __restrict__ row_loss, const float* __restrict__ weight, const int32_t* __restrict__ count, float* __restrict__ loss, int n) {
  __shared__ float red[17];
  float s = 0.f;
  auto add = [&](float l, float g) { s += l != 0.f ? g * l : 0.f; };
  int t = threadIdx.x;
  for (; t + 7 * 1024 < n; t += 8 * 1024) {          // eight loads in flight
    float l[8], g[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) { l[k] = row_loss[t + 1024 * k]; g[k] = weight ? weight[t + 1024 * k] : 1.f; }
#pragma unroll
    for (int k = 0; k < 8; ++k) add(l[k], g[k]);
  }
  for (; t < n; t += 1024) add(row_loss[t], weight ? weight[t] : 1.f);
  s = block_sum(s, red);
  if (threadIdx.x == 0) *loss = weight ? s : s / (float)max(*count, 1);
}

// ------------------------------------------------------------------------------------------------ one call
static dim3 quads(int rows) { return dim3((rows + 3) / 4); }

template <class T, int NT>
static void few_grads(hipStream_t st, const HeadArgs& a, HeadFew h) {
  const int cols = few_cols(a.d), waves = few_waves(a.d), rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  const int slice = NT == 1 ? cols * 8 : waves * 128, slices = (a.d + slice - 1) / slice;
  h.chunk = few_chunk(a.vocab, a.d, a.n);
  h.chunk_dw = std::max(1, std::min(128, (int)(((long)rows * slices + 1023) / 1024)));
  if (NT > 1) h.chunk_dw = (h.chunk_dw + 15) / 16 * 16;
  const int groups = a.dx ? (a.vocab + h.chunk - 1) / h.chunk : 0;
  const dim3 grid(groups + (rows + h.chunk_dw - 1) / h.chunk_dw, slices);
  if (a.dw_f32) head_few_grads_kernel<T, float, NT><<<grid, 256, 0, st>>>(h, cols, waves, groups);
  else head_few_grads_kernel<T, T, NT><<<grid, 256, 0, st>>>(h, cols, waves, groups);
  if (a.dx) head_few_sum_kernel<T><<<dim3((a.d + 63) / 64, a.n), 1024, 0, st>>>(h, groups);
}
template <class T>
static void head_few(hipStream_t st, const HeadArgs& a, const HeadPlan& p, char* ws, float* row_loss) {
  HeadFew h{a.x, a.w, a.ldx, a.ldw, a.n, a.vocab, a.d, p.vp, p.parts, a.top, a.dw_lo, a.dw_hi, a.lddx, a.lddw, a.dw_f32 == 2, 0, 0, a.targets, a.ids, a.logits, a.row_weight, a.tau, a.share,
            (float*)(ws + p.z), (float*)(ws + p.stats), (float*)(ws + p.coef), (float*)(ws + p.scale), (float*)(ws + p.part), (int32_t*)(ws + p.zsel), a.loss, row_loss, a.row_lse, a.dx, a.dw};
  if (few_split((a.vocab + 15) / 16, a.d)) head_few_z_kernel<T, true><<<p.parts / 4, 256, 0, st>>>(h);
  else head_few_z_kernel<T, false><<<p.parts / 4, 256, 0, st>>>(h);
  head_few_fin_kernel<<<1, 1024, 0, st>>>(h);
  if (!a.dx && !a.dw) return;
  if (a.n == 1) few_grads<T, 1>(st, a, h);
  else if (a.n <= 4) few_grads<T, 4>(st, a, h);
  else if (a.n <= 8) few_grads<T, 8>(st, a, h);
  else few_grads<T, 16>(st, a, h);
}

static void head_f32(hipStream_t st, const HeadArgs& a, const HeadPlan& p, char* ws, const void* w, int ldw, const void* wt, int ldwt, float* row_loss) {
  const int dw_rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  auto* rows = (int32_t*)(ws + p.rows);
  auto* count = (int32_t*)(ws + p.count);
  float *z = (float*)(ws + p.z), *part = (float*)(ws + p.part);
  HeadRow h{rows, count, a.targets, a.ids, a.logits, a.row_weight, a.top ? (unsigned char*)(ws + p.flags) : nullptr, row_loss, a.row_lse, a.tau, a.share, a.vocab, p.vp, a.top, 0};
  for (int i0 = 0; i0 < a.n; i0 += p.piece) {
    const int m = std::min(p.piece, p.np - i0);
    const float* xp = (const float*)(ws + p.xc) + (size_t)i0 * p.dp;
    h.i0 = i0;
    k_gemm_nt_f32(st, 0, xp, p.dp, w, ldw, z, p.vp, m, a.vocab, a.d, EPI_STORE, nullptr, 1, 1, nullptr, count, i0, m);
    const int g = p.grads;
    if (p.vp <= 2 * 4 * 256) head_row_kernel<256, 2><<<m, 256, 0, st>>>(z, g, h);
    else if (p.vp <= 8 * 4 * 256) head_row_kernel<256, 8><<<m, 256, 0, st>>>(z, g, h);
    else if (p.vp <= 8 * 4 * 1024) head_row_kernel<1024, 8><<<m, 1024, 0, st>>>(z, g, h);
    else head_row_kernel<1024, 0><<<m, 1024, 0, st>>>(z, g, h);
    if (a.dx) {
      k_gemm_nt_f32(st, 0, z, p.vp, wt, ldwt, part, a.d, m, a.d, p.vp, EPI_STORE, nullptr, 1, p.dx_splits, part, count, i0, m);
      head_dx_sum_kernel<float><<<row_grid(m, a.d), 256, 0, st>>>(part, p.dx_splits, nullptr, m, nullptr, (float*)a.dx, a.lddx, a.d, rows, count, i0, m, row_lanes(a.d));
    }
    if (a.dw) {
      // (columns too long for the kernel's offsets cannot happen: vp < 2^20 + 128)
      const bool add = i0 > 0 || a.dw_f32 == 2;
      float* dw = (float*)a.dw;
      if (p.dw_splits == 1 && !add) k_gemm_tn_f32(st, z + a.dw_lo, p.vp, dw_rows, 0, xp, p.dp, dw, a.lddw, dw_rows, a.d, m, 1, nullptr, count, i0, m);
      else {
        const int splits = m % (4 * p.dw_splits) == 0 ? p.dw_splits : 1;
        k_gemm_tn_f32(st, z + a.dw_lo, p.vp, dw_rows, 0, xp, p.dp, part, a.d, dw_rows, a.d, m, splits, part, count, i0, m);
        head_dw_sum_kernel<float><<<row_grid(dw_rows, a.d), 256, 0, st>>>(part, splits, add ? dw : nullptr, a.lddw, dw, a.lddw, dw_rows, a.d, row_lanes(a.d));
      }
    }
  }
}

static bool head_bf16(hipStream_t st, const HeadArgs& a, const HeadPlan& p, char* ws, const void* w, int ldw, float* row_loss) {
  const int dw_rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  auto* rows = (int32_t*)(ws + p.rows);
  auto* count = (int32_t*)(ws + p.count);
  auto* flags = a.top ? (unsigned char*)(ws + p.flags) : nullptr;
  float *ref = (float*)(ws + p.ref), *scale = (float*)(ws + p.scale), *zsel = (float*)(ws + p.zsel), *part = (float*)(ws + p.part);
  auto* stats = (float2*)(ws + p.stats);
  auto* stats2 = (float*)(ws + p.stats2);
  auto* coef = p.mixed ? (float2*)(ws + p.coef) : nullptr;
  bf16_t* e = p.grads ? (bf16_t*)(ws + p.z) : nullptr;
  const bf16_t* xc = (const bf16_t*)(ws + p.xc);
  bool ok = true;
  const int group = p.pick ? 1 : p.ref_group;
  head_ref_kernel<<<dim3((p.np + 3) / 4, p.pick ? 1 : std::max(1, (a.top + group - 1) / group)), 256, 0, st>>>(HeadRef{(const bf16_t*)a.x, (const bf16_t*)w, (bf16_t*)(ws + p.xc), (bf16_t*)a.dx, a.ldx, ldw, a.lddx, a.d, p.dp, a.n, p.np, a.vocab, a.top,
                                                       a.ldx % 8 == 0 && ((uintptr_t)a.x & 15) == 0, group, (const int32_t*)(ws + p.pos), count, a.targets, a.ids, a.logits, flags, zsel, ref, row_loss, a.row_lse});
  const float log2e = 1.44269504f;
  for (int i0 = 0; i0 < a.n; i0 += p.piece) {
    const int m = std::min(p.piece, p.np - i0);          // a multiple of 64
    const bf16_t* xp = xc + (size_t)i0 * p.dp;
    auto* redo = (int32_t*)(ws + p.redo) + (size_t)(i0 / p.piece) * (1 + (p.piece + 255) / 256);
    HeadEpi he{};
    he.count = count; he.i0 = i0; he.piece = m; he.ref = ref; he.stats = stats; he.stats2 = stats2; he.k = p.mixed ? log2e : log2e / a.tau; he.kt = p.mixed ? log2e / a.tau : 0.f; he.vp = p.vp; he.tile = p.exp_tile;
    if (p.pick) {
      const int groups64 = (a.vocab + 255) / 256 * 4;
      head_lists_kernel<<<(m + 127) / 128, 1024, groups64 * 4, st>>>(rows, count, a.ids, a.logits, flags, a.vocab, a.top, i0, m, groups64, (int32_t*)(ws + p.offs), (int32_t*)(ws + p.list));
      he.offs = (const int32_t*)(ws + p.offs); he.list = (const int32_t*)(ws + p.list); he.zsel = zsel; he.top = a.top;
    }
    he.own = !e && p.exp_tile;          // losses alone need no reference beforehand: no second launches (on 256 x 256 tiles the longer epilogue costs as much as those)
    HeadFin f{stats, stats2, p.groups, m, i0, a.vocab, p.vp, a.top, p.mixed, 0, rows, count, a.targets, a.ids, a.logits, a.row_weight, zsel, flags, ref, scale, row_loss, a.row_lse, coef, e,
              !p.mixed, redo, a.tau, a.share, he.k, he.kt};
    ok &= k_head_gemm(st, EPI_HEAD_EXP, xp, p.dp, w, ldw, e, p.vp, m, a.vocab, p.dp, p.dp, 1, he) == 0;
    if (he.own) {
      head_fin_kernel<true><<<m / 16, 1024, 0, st>>>(f);
      continue;
    }
    head_fin_kernel<false><<<m / 16, 1024, 0, st>>>(f);
    he.redo = redo; he.offs = nullptr;          // the logits are picked already
    f.again = 1;
    ok &= k_head_gemm(st, EPI_HEAD_EXP, xp, p.dp, w, ldw, e, p.vp, m, a.vocab, p.dp, p.dp, 1, he) == 0;
    head_fin_kernel<false><<<m / 16, 1024, 0, st>>>(f);
    if (!e) continue;
    if (p.mixed) {
      head_mix_kernel<<<dim3(m, (p.vp / 8 + 1023) / 1024), 256, 0, st>>>(e, p.vp, coef, count, i0, m, std::min(1.f, a.tau), std::min(1.f, 1.f / a.tau));
      f.again = 0; f.places = 1;
      head_fin_kernel<false><<<m / 16, 1024, 0, st>>>(f);
    }
    he.scale = scale; he.rows = rows;
    if (a.dx) {
      he.ncols = p.dp;          // of W: d where that is a multiple of 64, else of its padded copy
      he.splits = (const int32_t*)(ws + p.redo) + p.n_redo + i0 / p.piece;
      if (p.dx_whole) ok &= k_head_gemm(st, EPI_HEAD_DX, e, p.vp, w, ldw, a.dx, a.lddx, m, a.d, p.vp, a.vocab, 1, he) == 0;
      if (p.dx_splits > 1) {
        ok &= k_head_gemm(st, EPI_HEAD_PART, e, p.vp, w, ldw, part, a.d, m, a.d, p.vp, a.vocab, p.dx_splits, he) == 0;
        head_dx_sum_kernel<bf16_t><<<row_grid(m, a.d), 256, 0, st>>>(part, 0, he.splits, 0, scale, (bf16_t*)a.dx, a.lddx, a.d, rows, count, i0, m, row_lanes(a.d));
      }
    }
    if (a.dw) {
      const bool first = i0 == 0, last = i0 + p.piece >= a.n;
      const int v0 = a.dw_lo & ~7;          // columns of e are read in aligned groups of 8
      bf16_t* xt = (bf16_t*)(ws + p.xt);
      head_xt_kernel<<<dim3(m / 64, p.dp / 64), 256, 0, st>>>(xp, p.dp, scale, xt, p.piece, a.d, count, i0, m);
      // the sums of several pieces are kept in fp32: in dw itself where that is float, else in the workspace until the last
      float* acc = a.dw_f32 ? (float*)a.dw : (float*)(ws + p.dwa);
      const int ldacc = a.dw_f32 ? a.lddw : a.d;
      he.shift = a.dw_lo - v0; he.out_rows = dw_rows; he.ncols = p.vp - v0;
      he.add = !first || a.dw_f32 == 2 ? acc : nullptr; he.ldadd = ldacc;
      he.out_f32 = a.dw_f32 || !last;
      void* out = he.out_f32 ? (void*)acc : a.dw;
      const int ldo = he.out_f32 ? ldacc : a.lddw;
      if (p.dw_splits == 1)
        ok &= k_head_gemm(st, EPI_HEAD_DW, xt, p.piece, e + v0, p.vp, out, ldo, a.d, a.dw_hi - v0, m, m, 1, he) == 0;
      else {
        ok &= k_head_gemm(st, EPI_HEAD_DW_PART, xt, p.piece, e + v0, p.vp, part, a.d, a.d, a.dw_hi - v0, m, m, p.dw_splits, he) == 0;
        if (he.out_f32) head_dw_sum_kernel<float><<<row_grid(dw_rows, a.d), 256, 0, st>>>(part, p.dw_splits, he.add, ldacc, (float*)out, ldo, dw_rows, a.d, row_lanes(a.d));
        else head_dw_sum_kernel<bf16_t><<<row_grid(dw_rows, a.d), 256, 0, st>>>(part, p.dw_splits, he.add, ldacc, (bf16_t*)out, ldo, dw_rows, a.d, row_lanes(a.d));
      }
    }
  }
  return ok;
}

int k_head(hipStream_t st, const HeadArgs& a, char* ws) {
  const HeadPlan p = plan_head(a);
  const int dw_rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  auto* pos = (int32_t*)(ws + p.pos);
  auto* rows = (int32_t*)(ws + p.rows);
  auto* count = (int32_t*)(ws + p.count);
  auto* flags = a.top ? (unsigned char*)(ws + p.flags) : nullptr;
  float* row_loss = a.row_loss ? a.row_loss : (float*)(ws + p.rowl);
  char* xc = ws + p.xc;

  if (p.parts) {
    PP_H_DISPATCH(a.dtype, head_few<T>(st, a, p, ws, row_loss));
    return 0;
  }
  if (a.top && a.n) head_flags_kernel<<<quads(a.n), 256, 0, st>>>(a.targets, a.ids, a.logits, a.row_weight, flags, a.n, a.vocab, a.top, a.share > 0.f);
  head_scan_kernel<<<1, 1024, 0, st>>>(a.targets, flags, a.row_weight, a.n, a.vocab, pos, rows, count, (int32_t*)(ws + p.redo), p.n_redo,
                                      a.dtype && a.dx ? (p.np + p.piece - 1) / p.piece : 0, p.piece, (a.d + 255) / 256, p.vp / 64, p.dx_splits, a.part_cap, a.d);
  if (a.dtype == 0)
    head_gather_kernel<<<quads(p.np), 256, 0, st>>>((const float*)a.x, a.ldx, (float*)xc, p.dp, a.d, pos, count, a.n, p.np, (float*)a.dx, a.lddx, row_loss, a.row_lse);
  const void* w = a.w;
  int ldw = a.ldw;
  if (p.copy_w) {
    head_pad_kernel<<<quads(a.vocab), 256, 0, st>>>((const bf16_t*)a.w, a.ldw, (bf16_t*)(ws + p.wc), p.dp, a.vocab, a.d);
    w = ws + p.wc; ldw = p.dp;
  }
  const void* wt = a.wt;
  int ldwt = a.ldwt;
  if (p.own_wt) {
    head_transpose_kernel<<<dim3((p.vp + 63) / 64, (a.d + 63) / 64), 256, 0, st>>>((const float*)a.w, a.ldw, (float*)(ws + p.wt), p.vp, a.vocab, a.d);
    wt = ws + p.wt; ldwt = p.vp;
  }
  if (a.n == 0 && a.dw && a.dw_f32 != 2) {
    if (a.dw_f32) head_zero_kernel<float><<<quads(dw_rows), 256, 0, st>>>((float*)a.dw, a.lddw, dw_rows, a.d);
    else PP_H_DISPATCH(a.dtype, head_zero_kernel<T><<<quads(dw_rows), 256, 0, st>>>((T*)a.dw, a.lddw, dw_rows, a.d));
  }
  bool ok = true;
  if (a.dtype) ok = head_bf16(st, a, p, ws, w, ldw, row_loss);
  else head_f32(st, a, p, ws, w, ldw, wt, ldwt, row_loss);
  if (a.loss) head_loss_kernel<<<1, 1024, 0, st>>>(row_loss, a.row_weight, count, a.loss, a.n);
  return ok ? 0 : 1;
}

}  // namespace pp
