// Losses of the output head (cross entropy, distillation from a teacher's top logits) with their gradients, the logits existing a piece of rows at a time.
//
// With z = X W^T:  dz_tv = g_t [ c1 (p_tv - [v = y_t]) + ct (pt_tv - Q_tv) ],  p = softmax(z), pt = softmax(z / tau), c1 = 1 - share (rows with a target), ct = share tau (rows
// with entries), Q the teacher's q at its entries;  dX = dz W,  dW = dz^T X.
// Rows that count are gathered into the front of the workspace's copy of X, whose rows are padded with zeros to what the matrix kernels read; every
// kernel below works on those compact rows, in pieces.
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
  int dp, vp, np, piece;          // padded width, padded vocabulary, rows of the compact X, rows of a piece
  bool grads, copy_w, own_wt;
  size_t flags, pos, rows, count, rowl, xc, wc, wt, z, dz, dzt, xt, dxc, dwa, dwp, total;          // byte offsets
};
int pad_to(long v, int m) { return (int)((v + m - 1) / m * m); }

HeadPlan plan_head(const HeadArgs& a) {
  HeadPlan p{};
  const size_t es = a.dtype == 0 ? 4 : 2;
  const int unit = a.dtype == 0 ? 4 : 64;
  const size_t dw_rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  p.grads = a.dx || a.dw;
  p.dp = pad_to(a.d, unit);
  p.vp = pad_to(a.vocab, unit);
  p.np = std::max(64, pad_to(a.n, 64));
  const size_t row = (size_t)p.vp * es;
  p.piece = a.piece ? pad_to(a.piece, 64) : std::max(256, (int)(kPieceBytes / row / 256 * 256));
  p.piece = std::min(p.piece, p.np);
  // the bf16 matrix kernels read rows that are multiples of 64 elements long and 16-byte aligned, the fp32 ones any
  p.copy_w = a.dtype != 0 && (a.d % 64 || a.ldw % 8 || (uintptr_t)a.w & 15);
  p.own_wt = a.dx && !(a.wt && a.vocab % unit == 0 && a.ldwt % 8 == 0 && ((uintptr_t)a.wt & 15) == 0);
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
  p.z = take((size_t)p.piece * p.vp * 4);
  p.dz = take(p.grads && a.dtype ? (size_t)p.piece * p.vp * es : 0);          // fp32: in place of z
  p.dzt = take(a.dw && a.dtype ? dw_rows * p.piece * es : 0);
  p.xt = take(a.dw && a.dtype ? (size_t)a.d * p.piece * es : 0);
  p.dxc = take(a.dx ? (size_t)p.piece * p.dp * es : 0);
  p.dwa = take(dw_rows * a.d * 4);
  p.dwp = take(p.piece < a.n ? dw_rows * a.d * 4 : 0);
  p.total = off;
  return p;
}
}  // namespace
size_t head_bytes(const HeadArgs& a) { return plan_head(a).total; }

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

// pos[t] = place of row t among the rows that count, -1 for the others; rows[i] = t; count = their number.  One block; 16 consecutive rows per thread.
__global__ __launch_bounds__(1024) void head_scan_kernel(const int32_t* __restrict__ targets, const unsigned char* __restrict__ flags, const float* __restrict__ weight, int n, int V,
                                                         int32_t* __restrict__ pos, int32_t* __restrict__ rows, int32_t* __restrict__ count) {
  __shared__ int wave_sum_s[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int base = 0;
  for (int t0 = 0; t0 < n; t0 += 16 * 1024) {
    const int first = t0 + tid * 16;
    uint32_t live = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int t = first + e;
      if (t < n && (flags ? flags[t] != 0 : hard_row(targets, t, V) && !(weight && weight[t] == 0.f))) live |= 1u << e;
    }
    const int mine = __popc(live);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 63) wave_sum_s[wave] = incl;
    __syncthreads();
    int before = base, all = 0;
    for (int w = 0; w < 16; ++w) { if (w < wave) before += wave_sum_s[w]; all += wave_sum_s[w]; }
    int at = before + incl - mine;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int t = first + e;
      if (t >= n) break;
      const bool l = live >> e & 1;
      pos[t] = l ? at : -1;
      if (l) rows[at++] = t;
    }
    base += all;
  }
  if (tid == 0) *count = base;
}

// Compact, padded copy of the rows that count; zeros behind them up to the last row of the copy; the outputs of rows that are left out.  A wave per row.
template <class T>
__global__ __launch_bounds__(256) void head_gather_kernel(const T* __restrict__ x, int ldx, T* __restrict__ xc, int dp, int d, const int32_t* __restrict__ pos, const int32_t* __restrict__ count,
                                                          int n, int np, T* __restrict__ dx, int lddx, float* __restrict__ row_loss, float* __restrict__ row_lse) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= np) return;
  if (t >= *count)
    for (int c = lane; c < dp; c += 64) xc[(size_t)t * dp + c] = from_f32<T>(0.f);
  if (t >= n) return;
  const int i = pos[t];
  if (i < 0) {
    if (dx) for (int c = lane; c < d; c += 64) dx[(size_t)t * lddx + c] = from_f32<T>(0.f);
    if (lane == 0) { row_loss[t] = 0.f; if (row_lse) row_lse[t] = 0.f; }
    return;
  }
  for (int c = lane; c < dp; c += 64) xc[(size_t)i * dp + c] = c < d ? x[(size_t)t * ldx + c] : from_f32<T>(0.f);
}

// dst [rows x ld_dst] = src [rows x cols], zeros from column cols to ld_dst
template <class T>
__global__ __launch_bounds__(256) void head_pad_kernel(const T* __restrict__ src, int ld_src, T* __restrict__ dst, int ld_dst, int rows, int cols) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  for (int c = threadIdx.x & 63; c < ld_dst; c += 64) dst[(size_t)r * ld_dst + c] = c < cols ? src[(size_t)r * ld_src + c] : from_f32<T>(0.f);
}
// dst[c][r] = src[r][c] for r < rows, zeros for rows <= r < ld_dst
template <class T>
__global__ __launch_bounds__(256) void head_transpose_kernel(const T* __restrict__ src, int ld_src, T* __restrict__ dst, int ld_dst, int rows, int cols) {
  __shared__ T tile[64][65];
  const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  for (int i = ty; i < 64; i += 4) tile[i][tx] = r0 + i < rows && c0 + tx < cols ? src[(size_t)(r0 + i) * ld_src + c0 + tx] : from_f32<T>(0.f);
  __syncthreads();
  for (int i = ty; i < 64; i += 4)
    if (c0 + i < cols && r0 + tx < ld_dst) dst[(size_t)(c0 + i) * ld_dst + r0 + tx] = tile[tx][i];
}

// ------------------------------------------------------------------------------------------------ softmax, losses and dz of a row of logits
// One block per compact row of the piece.  z [piece x vp] fp32; dz [piece x vp] in storage type (may be z itself) or nullptr.  Rows from *count on get zeros.
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
    if ((uint32_t)id < (uint32_t)h.V) u = h.logits[(size_t)t * h.top + j] / h.tau; else id = -1;
    if (u == -INFINITY) id = -1;
  }
  // NaN among the entries has to reach the sum: fmaxf would drop it from the maximum
  const float m = block_max(id >= 0 ? u : -INFINITY, red);
  const float e = id >= 0 ? expf(u - m) : 0.f;
  const float s = block_sum(e, red);
  if (j < h.top) { id_s[j] = id; q_s[j] = id >= 0 ? e / s : 0.f; }
  __syncthreads();
}

template <class T>
__global__ __launch_bounds__(256) void head_row_kernel(const float* z_, T* dz_, HeadRow h) {
  __shared__ float red[17];
  __shared__ int id_s[kTopMax];
  __shared__ float q_s[kTopMax];
  const int i = h.i0 + blockIdx.x, tid = threadIdx.x, n_live = *h.count;
  const float* z = z_ + (size_t)blockIdx.x * h.vp;
  T* dz = dz_ ? dz_ + (size_t)blockIdx.x * h.vp : nullptr;
  if (i >= n_live) {
    if (dz) for (int v = tid; v < h.vp; v += 256) dz[v] = from_f32<T>(0.f);
    return;
  }
  const int t = h.rows[i];
  const bool hard = h.flags ? h.flags[t] & ROW_HARD : true, soft = h.flags ? h.flags[t] & ROW_SOFT : false;
  const float it = 1.0f / h.tau;
  float m = -INFINITY;
  for (int v = tid; v < h.V; v += 256) m = fmaxf(m, z[v]);
  m = block_max(m, red);
  float s1 = 0.f, st = 0.f;
  for (int v = tid; v < h.V; v += 256) {
    s1 += expf(z[v] - m);
    if (h.tau != 1.f) st += expf((z[v] - m) * it);
  }
  s1 = block_sum(s1, red);
  st = h.tau != 1.f ? block_sum(st, red) : s1;
  if (soft) head_entries(h, t, id_s, q_s, red);
  const int y = hard ? h.targets[t] : -1;
  // losses
  float kl = 0.f;
  if (soft && tid < h.top && id_s[tid] >= 0 && !(q_s[tid] <= 0.f)) kl = q_s[tid] * (logf(q_s[tid]) - (z[id_s[tid]] - m) * it + logf(st));
  kl = block_sum(kl, red);
  if (tid == 0) {
    float l = soft ? h.share * h.tau * h.tau * kl : 0.f;
    if (hard) l += (1.f - h.share) * ((m - z[y]) + logf(s1));
    h.row_loss[t] = l;
    if (h.row_lse) h.row_lse[t] = m * it + logf(st);
  }
  if (!dz) return;
  const float g = h.weight ? h.weight[t] : 1.0f / (float)max(n_live, 1);
  const float c1 = hard ? g * (1.f - h.share) : 0.f, ct = soft ? g * h.share * h.tau : 0.f;
  const float p1 = c1 / s1, pt = ct / st;
  auto soft_part = [&](float zv) { return (c1 != 0.f ? p1 * expf(zv - m) : 0.f) + (ct != 0.f ? pt * expf((zv - m) * it) : 0.f); };
  // entry j of the row, or the target (j == top): its part of dz is formed from z before the row may be overwritten (dz may be z).  The first of equal
  // ids stores the sum of all, in their order.
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
  for (int v = tid; v < h.vp; v += 256) dz[v] = from_f32<T>(v < h.V ? soft_part(z[v]) : 0.f);
  __syncthreads();
  if (at >= 0) dz[at] = from_f32<T>(own);
}

// ------------------------------------------------------------------------------------------------ outputs
// dx[rows[i]] = dxc[i] for the compact rows of a piece
template <class T>
__global__ __launch_bounds__(256) void head_scatter_kernel(const T* __restrict__ dxc, int dp, T* __restrict__ dx, int lddx, int d, const int32_t* __restrict__ rows, const int32_t* __restrict__ count,
                                                           int i0, int m) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= m || i0 + i >= *count) return;
  const int t = rows[i0 + i];
  for (int c = threadIdx.x & 63; c < d; c += 64) dx[(size_t)t * lddx + c] = dxc[(size_t)i * dp + c];
}
// out (+)= acc, rows of d; or, with `sum`, sum (+)= acc
template <class TO>
__global__ __launch_bounds__(256) void head_add_kernel(const float* __restrict__ acc, TO* out, int ldo, int rows, int d, int add) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  for (int c = threadIdx.x & 63; c < d; c += 64) {
    TO* o = out + (size_t)r * ldo + c;
    const float v = acc ? acc[(size_t)r * d + c] : 0.f;
    *o = from_f32<TO>(add ? to_f32(*o) + v : v);
  }
}
__global__ __launch_bounds__(1024) void head_loss_kernel(const float* __restrict__ row_loss, const float* __restrict__ weight, const int32_t* __restrict__ pos, const int32_t* __restrict__ count,
                                                         float* __restrict__ loss, int n) {
  __shared__ float red[17];
  float s = 0.f;
  for (int t = threadIdx.x; t < n; t += 1024)
    if (pos[t] >= 0) s += weight ? weight[t] * row_loss[t] : row_loss[t];
  s = block_sum(s, red);
  if (threadIdx.x == 0) *loss = weight ? s : s / (float)max(*count, 1);
}

// ------------------------------------------------------------------------------------------------ one call
int k_head(hipStream_t st, const HeadArgs& a, char* ws) {
  const HeadPlan p = plan_head(a);
  const int dw_rows = a.dw ? a.dw_hi - a.dw_lo : 0;
  const size_t es = a.dtype == 0 ? 4 : 2;
  auto quads = [](int rows) { return dim3((rows + 3) / 4); };
  auto* pos = (int32_t*)(ws + p.pos);
  auto* rows = (int32_t*)(ws + p.rows);
  auto* count = (int32_t*)(ws + p.count);
  auto* flags = a.top ? (unsigned char*)(ws + p.flags) : nullptr;
  auto* dwa = (float*)(ws + p.dwa);
  float* row_loss = a.row_loss ? a.row_loss : (float*)(ws + p.rowl);
  char* xc = ws + p.xc;

  if (a.top && a.n) head_flags_kernel<<<quads(a.n), 256, 0, st>>>(a.targets, a.ids, a.logits, a.row_weight, flags, a.n, a.vocab, a.top, a.share > 0.f);
  head_scan_kernel<<<1, 1024, 0, st>>>(a.targets, flags, a.row_weight, a.n, a.vocab, pos, rows, count);
  PP_H_DISPATCH(a.dtype, head_gather_kernel<T><<<quads(p.np), 256, 0, st>>>((const T*)a.x, a.ldx, (T*)xc, p.dp, a.d, pos, count, a.n, p.np, (T*)a.dx, a.lddx, row_loss, a.row_lse));
  const void* w = a.w;
  int ldw = a.ldw;
  if (p.copy_w) {
    PP_H_DISPATCH(a.dtype, head_pad_kernel<T><<<quads(a.vocab), 256, 0, st>>>((const T*)a.w, a.ldw, (T*)(ws + p.wc), p.dp, a.vocab, a.d));
    w = ws + p.wc; ldw = p.dp;
  }
  const void* wt = a.wt;
  int ldwt = a.ldwt;
  auto transpose = [&](const void* src, int ld_src, void* dst, int ld_dst, int r, int c) {
    PP_H_DISPATCH(a.dtype, head_transpose_kernel<T><<<dim3((ld_dst + 63) / 64, (c + 63) / 64), 256, 0, st>>>((const T*)src, ld_src, (T*)dst, ld_dst, r, c));
  };
  if (p.own_wt) { transpose(a.w, a.ldw, ws + p.wt, p.vp, a.vocab, a.d); wt = ws + p.wt; ldwt = p.vp; }

  HeadRow h{rows, count, a.targets, a.ids, a.logits, a.row_weight, flags, row_loss, a.row_lse, a.tau, a.share, a.vocab, p.vp, a.top, 0};
  bool ok = true;
  if (a.n == 0 && a.dw && a.dw_f32 != 2) {
    if (a.dw_f32) head_add_kernel<float><<<quads(dw_rows), 256, 0, st>>>(nullptr, (float*)a.dw, a.lddw, dw_rows, a.d, 0);
    else PP_H_DISPATCH(a.dtype, head_add_kernel<T><<<quads(dw_rows), 256, 0, st>>>(nullptr, (T*)a.dw, a.lddw, dw_rows, a.d, 0));
  }
  for (int i0 = 0; i0 < a.n; i0 += p.piece) {
    const int m = std::min(p.piece, p.np - i0);          // a multiple of 64
    const char* xp = xc + (size_t)i0 * p.dp * es;
    float* z = (float*)(ws + p.z);
    char* dz = a.dtype ? ws + p.dz : ws + p.z;
    h.i0 = i0;
    auto nt = [&](const void* A, int lda, const void* B, int ldb, void* C, int ldc, int M, int N, int K, int out_f32) {
      if (a.dtype) ok &= k_gemm_nt_mfma(st, A, lda, B, ldb, C, ldc, M, N, K, EPI_STORE, nullptr, out_f32, 1, nullptr) == 0;
      else k_gemm_nt_f32(st, 0, A, lda, B, ldb, C, ldc, M, N, K, EPI_STORE, nullptr, 1, 1, nullptr);
    };
    nt(xp, p.dp, w, ldw, z, p.vp, m, a.vocab, a.dtype ? p.dp : a.d, 1);
    PP_H_DISPATCH(a.dtype, head_row_kernel<T><<<m, 256, 0, st>>>(z, p.grads ? (T*)dz : nullptr, h));
    if (a.dx) {
      nt(dz, p.vp, wt, ldwt, ws + p.dxc, p.dp, m, a.d, a.dtype ? p.vp : a.vocab, 0);
      PP_H_DISPATCH(a.dtype, head_scatter_kernel<T><<<quads(m), 256, 0, st>>>((const T*)(ws + p.dxc), p.dp, (T*)a.dx, a.lddx, a.d, rows, count, i0, m));
    }
    if (a.dw) {
      const char* dzs = dz + (size_t)a.dw_lo * es;
      const bool first = i0 == 0, last = i0 + p.piece >= a.n;
      float* prod = first ? dwa : (float*)(ws + p.dwp);
      if (a.dtype) {
        transpose(dzs, p.vp, ws + p.dzt, p.piece, m, dw_rows);
        transpose(xp, p.dp, ws + p.xt, p.piece, m, a.d);
        nt(ws + p.dzt, p.piece, ws + p.xt, p.piece, prod, a.d, dw_rows, a.d, m, 1);
      } else
        ok &= k_gemm_tn_f32(st, (const float*)dzs, p.vp, dw_rows, 0, (const float*)xp, p.dp, prod, a.d, dw_rows, a.d, m, 1, nullptr) == 0;
      if (!first) head_add_kernel<float><<<quads(dw_rows), 256, 0, st>>>(prod, dwa, a.d, dw_rows, a.d, 1);
      if (last) {
        if (a.dw_f32) head_add_kernel<float><<<quads(dw_rows), 256, 0, st>>>(dwa, (float*)a.dw, a.lddw, dw_rows, a.d, a.dw_f32 == 2);
        else PP_H_DISPATCH(a.dtype, head_add_kernel<T><<<quads(dw_rows), 256, 0, st>>>(dwa, (T*)a.dw, a.lddw, dw_rows, a.d, 0));
      }
    }
  }
  if (a.loss) head_loss_kernel<<<1, 1024, 0, st>>>(row_loss, a.row_weight, pos, count, a.loss, a.n);
  return ok ? 0 : 1;
}

}  // namespace pp
