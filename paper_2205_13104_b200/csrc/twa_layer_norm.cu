// Layer norm of rows and its gradient.
//
//   forward    mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps),
//              y = (x - mean) rstd w + b
//   backward   h = (x - mean) rstd,  v = dy w,
//              dx = rstd (v - sum v / cols - h sum(v h) / cols),   dw = sum_rows dy h,   db = sum_rows dy
//
// Both are bound by memory: a pass over x (and dy) and one store.  A row stays in the registers of the threads that
// share it, so it is read once, and the variance is taken from the differences to the mean, in a second
// reduction over registers: a sum of squares would lose the digits that a mean far from zero costs.
// A thread keeps the same columns for all rows of its block, and with them the weights and, backward, the columns'
// partial sums of dw and db, in float32 registers.  The partial sums of the blocks are added in float64 by a second
// kernel in block order, so results repeat bit for bit.
#include "twa_ops.cuh"

namespace {

constexpr int LN_MAX_BLOCKS = 592;     // blocks of the backward pass at most: rows of partial sums in the workspace
constexpr int LN_WARP_THREADS = 128;   // a warp per row, a block per row: threads at most
constexpr int LN_BLOCK_THREADS = 512;
constexpr int LN_LOOP_THREADS = 512;   // rows wider than the registers of a block

struct LnArgs {
  const void* x;
  const void* dy;      // backward
  void* y;             // forward: y; backward: dx
  const void* w;
  const void* b;
  float* mean;
  float* rstd;
  float* part;         // backward: [blocks][2][cols] partial sums of dw and db
  long long ldx, lddy, ldy, rows;
  int cols, w_dtype;
  float eps;
};

// Sum of N values over the threads that share a row: a warp, or the block (one barrier; `red` is used in turn
// by successive calls, two sets, so that a set is written again only after the next barrier).
template <bool WARP, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* red, int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = twa_warp_sum(v[i]);
  if (WARP) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  float* set = red + turn * 64;
  turn ^= 1;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) set[i * 32 + warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = twa_warp_sum(lane < warps ? set[i * 32 + lane] : 0.0f);
}

// NV packs of E elements per thread: columns (k * threads + thread) * E ...
template <typename T, int E, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? LN_WARP_THREADS : LN_BLOCK_THREADS) ln_forward_kernel(const LnArgs a) {
  __shared__ float red[128];
  int turn = 0;
  const int per = WARP ? 32 : blockDim.x;
  const int t = WARP ? (threadIdx.x & 31) : threadIdx.x;
  const long long first = WARP ? static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const long long step = WARP ? static_cast<long long>(gridDim.x) * (blockDim.x >> 5) : gridDim.x;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  float w[NV * E], b[NV * E];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (k * per + t) * E + e;
      w[k * E + e] = (a.w && c < a.cols) ? twa_load_any(a.w, a.w_dtype, c) : 1.0f;
      b[k * E + e] = (a.b && c < a.cols) ? twa_load_any(a.b, a.w_dtype, c) : 0.0f;
    }
  const float inv = 1.0f / static_cast<float>(a.cols);
  twa_pack<T, E> raw[NV] = {};
  if (first < a.rows)
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if ((k * per + t) * E < a.cols) raw[k].load(x + first * a.ldx + (k * per + t) * E);
  for (long long r = first; r < a.rows; r += step) {
    float v[NV * E];
    float s[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      raw[k].widen(v + k * E);
      if ((k * per + t) * E >= a.cols)
#pragma unroll
        for (int e = 0; e < E; ++e) v[k * E + e] = 0.0f;
    }
    if (r + step < a.rows)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if ((k * per + t) * E < a.cols) raw[k].load(x + (r + step) * a.ldx + (k * per + t) * E);
#pragma unroll
    for (int i = 0; i < NV * E; ++i) s[0] += v[i];
    row_sum<WARP>(s, red, turn);
    const float mean = s[0] * inv;
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if ((k * per + t) * E < a.cols)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          v[k * E + e] -= mean;
          q[0] += v[k * E + e] * v[k * E + e];
        }
    row_sum<WARP>(q, red, turn);
    const float rstd = 1.0f / sqrtf(q[0] * inv + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if ((k * per + t) * E < a.cols) {
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = v[k * E + e] * rstd * w[k * E + e] + b[k * E + e];
        twa_pack<T, E>::store(y + r * a.ldy + (k * per + t) * E, o);
      }
  }
}

template <typename T, int E, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? LN_WARP_THREADS : LN_BLOCK_THREADS) ln_backward_kernel(const LnArgs a) {
  extern __shared__ float sums[];      // WARP: the warps' partial sums of dw and db, [2][cols]
  __shared__ float red[128];
  int turn = 0;
  const int per = WARP ? 32 : blockDim.x;
  const int t = WARP ? (threadIdx.x & 31) : threadIdx.x;
  const long long first = WARP ? static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const long long step = WARP ? static_cast<long long>(gridDim.x) * (blockDim.x >> 5) : gridDim.x;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.y);
  float w[NV * E], dw[NV * E], db[NV * E];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (k * per + t) * E + e;
      w[k * E + e] = (a.w && c < a.cols) ? twa_load_any(a.w, a.w_dtype, c) : 1.0f;
      dw[k * E + e] = db[k * E + e] = 0.0f;
    }
  const float inv = 1.0f / static_cast<float>(a.cols);
  twa_pack<T, E> rx[NV] = {}, rd[NV] = {};
  float mean = 0.0f, rstd = 0.0f;
  if (first < a.rows) {
    mean = __ldg(a.mean + first);
    rstd = __ldg(a.rstd + first);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if ((k * per + t) * E < a.cols) {
        rx[k].load(x + first * a.ldx + (k * per + t) * E);
        rd[k].load(dy + first * a.lddy + (k * per + t) * E);
      }
  }
  for (long long r = first; r < a.rows; r += step) {
    float h[NV * E], v[NV * E];
    float s[2] = {0.0f, 0.0f};
    const float rs = rstd;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const bool in = (k * per + t) * E < a.cols;
      rx[k].widen(h + k * E);
      rd[k].widen(v + k * E);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = k * E + e;
        h[i] = in ? (h[i] - mean) * rs : 0.0f;
        const float d = in ? v[i] : 0.0f;
        dw[i] += d * h[i];
        db[i] += d;
        v[i] = d * w[i];
        s[0] += v[i];
        s[1] += v[i] * h[i];
      }
    }
    if (r + step < a.rows) {
      mean = __ldg(a.mean + r + step);
      rstd = __ldg(a.rstd + r + step);
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if ((k * per + t) * E < a.cols) {
          rx[k].load(x + (r + step) * a.ldx + (k * per + t) * E);
          rd[k].load(dy + (r + step) * a.lddy + (k * per + t) * E);
        }
    }
    row_sum<WARP>(s, red, turn);
    const float c1 = s[0] * inv, c2 = s[1] * inv;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if ((k * per + t) * E < a.cols) {
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = rs * (v[k * E + e] - c1 - h[k * E + e] * c2);
        twa_pack<T, E>::store(dx + r * a.ldy + (k * per + t) * E, o);
      }
  }
  if (!a.part) return;
  float* out = a.part + static_cast<long long>(blockIdx.x) * 2 * a.cols;
  if constexpr (!WARP) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = (k * per + t) * E + e;
        if (c < a.cols) {
          out[c] = dw[k * E + e];
          out[a.cols + c] = db[k * E + e];
        }
      }
  } else {
    // the warps add their sums in warp order
    for (int which = 0; which < static_cast<int>(blockDim.x >> 5); ++which) {
      if (which == static_cast<int>(threadIdx.x >> 5))
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int c = (k * per + t) * E + e;
            if (c < a.cols) {
              sums[c] = which ? sums[c] + dw[k * E + e] : dw[k * E + e];
              sums[a.cols + c] = which ? sums[a.cols + c] + db[k * E + e] : db[k * E + e];
            }
          }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * a.cols; c += blockDim.x) out[c] = sums[c];
  }
}

// Rows of any width, a block per row: the row is read again for each of its passes (from L2, while it fits there).
template <typename T>
__global__ void ln_forward_loop_kernel(const LnArgs a) {
  __shared__ float red[128];
  int turn = 0;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* xr = x + r * a.ldx;
    float s[1] = {0.0f};
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) s[0] += twa_to_float(xr[c]);
    row_sum<false>(s, red, turn);
    const float mean = s[0] / static_cast<float>(a.cols);
    float q[1] = {0.0f};
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float d = twa_to_float(xr[c]) - mean;
      q[0] += d * d;
    }
    row_sum<false>(q, red, turn);
    const float rstd = 1.0f / sqrtf(q[0] / static_cast<float>(a.cols) + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float w = a.w ? twa_load_any(a.w, a.w_dtype, c) : 1.0f, b = a.b ? twa_load_any(a.b, a.w_dtype, c) : 0.0f;
      y[r * a.ldy + c] = twa_from_float<T>((twa_to_float(xr[c]) - mean) * rstd * w + b);
    }
  }
}

template <typename T>
__global__ void ln_backward_loop_kernel(const LnArgs a) {
  __shared__ float red[128];
  int turn = 0;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.y);
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *xr = x + r * a.ldx, *dr = dy + r * a.lddy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.0f, 0.0f};
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float v = twa_to_float(dr[c]) * (a.w ? twa_load_any(a.w, a.w_dtype, c) : 1.0f);
      s[0] += v;
      s[1] += v * ((twa_to_float(xr[c]) - mean) * rstd);
    }
    row_sum<false>(s, red, turn);
    const float c1 = s[0] / static_cast<float>(a.cols), c2 = s[1] / static_cast<float>(a.cols);
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float v = twa_to_float(dr[c]) * (a.w ? twa_load_any(a.w, a.w_dtype, c) : 1.0f);
      const float h = (twa_to_float(xr[c]) - mean) * rstd;
      dx[r * a.ldy + c] = twa_from_float<T>(rstd * (v - c1 - h * c2));
    }
  }
}

// The columns' partial sums for those rows: a thread per column, blockIdx.y takes every gridDim.y-th row.
template <typename T>
__global__ void ln_weights_loop_kernel(const LnArgs a) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.cols) return;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  float dw = 0.0f, db = 0.0f;
  for (long long r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const float d = twa_to_float(dy[r * a.lddy + c]);
    dw += d * ((twa_to_float(x[r * a.ldx + c]) - a.mean[r]) * a.rstd[r]);
    db += d;
  }
  float* out = a.part + static_cast<long long>(blockIdx.y) * 2 * a.cols;
  out[c] = dw;
  out[a.cols + c] = db;
}

// Adds the blocks' partial sums in block order: 32 columns a block, its warps each a run of the blocks.
constexpr int LN_SUM_WARPS = 16;
__global__ void ln_sum_kernel(const float* __restrict__ part, int blocks, int cols, void* dw, void* db, int g_dtype,
                              int accumulate) {
  __shared__ double run[LN_SUM_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;               // 0 .. 2 cols: dw, then db
  const int each = (blocks + LN_SUM_WARPS - 1) / LN_SUM_WARPS;
  const int from = warp * each, to = min(blocks, from + each);
  double s = 0.0;
  if (c < 2 * cols)
    for (int k = from; k < to; ++k) s += static_cast<double>(__ldg(part + static_cast<long long>(k) * 2 * cols + c));
  run[warp][lane] = s;
  __syncthreads();
  if (warp || c >= 2 * cols) return;
  for (int k = 1; k < LN_SUM_WARPS; ++k) s += run[k][lane];
  void* out = c < cols ? dw : db;
  const int i = c < cols ? c : c - cols;
  if (!out) return;
  if (accumulate) s += static_cast<double>(twa_load_any(out, g_dtype, i));
  twa_store_any(out, g_dtype, i, static_cast<float>(s));
}

typedef void (*LnKernel)(const LnArgs);
struct LnPlan {
  LnKernel kernel;      // null: the rows do not fit in registers
  int threads, blocks;  // threads of a block
  size_t smem;
};

// What a thread holds of a row at most.  The backward pass holds x, dy, w and two sums per column.
constexpr int LN_FWD_HELD = 32, LN_BWD_HELD = 16;

template <typename T, int E, int NV, bool BACK>
LnKernel ln_pick(bool warp) {
  if constexpr (E * NV > (BACK ? LN_BWD_HELD : LN_FWD_HELD)) return nullptr;
  else if constexpr (BACK) return warp ? ln_backward_kernel<T, E, NV, true> : ln_backward_kernel<T, E, NV, false>;
  else return warp ? ln_forward_kernel<T, E, NV, true> : ln_forward_kernel<T, E, NV, false>;
}

template <typename T, int E, bool BACK>
LnKernel ln_pick_nv(bool warp, int nv) {
  if (nv <= 1) return ln_pick<T, E, 1, BACK>(warp);
  if (nv <= 2) return ln_pick<T, E, 2, BACK>(warp);
  if (nv <= 4) return ln_pick<T, E, 4, BACK>(warp);
  if (nv <= 8) return ln_pick<T, E, 8, BACK>(warp);
  if (nv <= 16) return ln_pick<T, E, 16, BACK>(warp);
  return ln_pick<T, E, 32, BACK>(warp);
}

template <typename T, bool BACK>
LnPlan ln_plan(const twa_ctx* ctx, bool packs, long long rows, int cols) {
  const int E = packs ? twa_vec<T> : 1;
  const int held = BACK ? LN_BWD_HELD : LN_FWD_HELD;
  const int units = (cols + E - 1) / E;
  LnPlan p = {nullptr, 0, 0, 0};
  const bool warp = units * E <= 32 * held;
  int nv;
  if (warp) {
    nv = (units + 31) / 32;
    p.threads = rows >= 4LL * ctx->sm_count ? LN_WARP_THREADS : 32;
  } else {
    nv = E < 8 ? 8 / E : 1;
    while (nv * E < held && (units + nv - 1) / nv > LN_BLOCK_THREADS / 2) nv *= 2;
    p.threads = ((units + nv - 1) / nv + 31) / 32 * 32;
    if (p.threads > LN_BLOCK_THREADS) return p;
  }
  p.kernel = packs ? ln_pick_nv<T, twa_vec<T>, BACK>(warp, nv) : ln_pick_nv<T, 1, BACK>(warp, nv);
  p.smem = BACK && warp ? sizeof(float) * 2 * cols : 0;
  const long long blocks = warp ? twa_ceil_div(rows, p.threads / 32) : rows;
  long long most = static_cast<long long>(ctx->sm_count) * (1024 / p.threads > 0 ? 1024 / p.threads : 1);
  if (BACK && most > LN_MAX_BLOCKS) most = LN_MAX_BLOCKS;
  p.blocks = static_cast<int>(blocks < most ? blocks : most);
  return p;
}

// Whether rows can be taken 16 bytes at a time.
bool ln_packs(const void* p, long long ld, int cols, size_t size) {
  return !twa_misaligned_to(p, 16) && (ld * size) % 16 == 0 && (cols * size) % 16 == 0;
}

int ln_check(const twa_ctx* ctx, twa_dtype dt, twa_dtype wt, int64_t rows, int cols) {
  if (!ctx || !twa_dtype_ok(dt) || !twa_dtype_ok(wt) || rows < 0 || cols < 1) return TWA_ERR_INVALID_ARG;
  if (rows > (1LL << 40) || cols > TWA_LAYER_NORM_MAX_COLS) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

}  // namespace

extern "C" {

size_t twa_layer_norm_workspace_bytes(int64_t rows, int cols) {
  if (rows < 0 || cols < 1) return 0;
  const long long blocks = rows < LN_MAX_BLOCKS ? (rows ? rows : 1) : LN_MAX_BLOCKS;
  return twa_round256(sizeof(float) * 2 * static_cast<size_t>(cols) * blocks);
}

int twa_layer_norm(twa_ctx* ctx, const void* x, int64_t ldx, twa_dtype dtype, const void* w, const void* b,
                   twa_dtype w_dtype, int64_t rows, int cols, float eps, void* y, int64_t ldy, float* mean, float* rstd) {
  int rc = ln_check(ctx, dtype, w_dtype, rows, cols);
  if (rc) return rc;
  if (rows == 0) return TWA_OK;
  if (!x || !y || ldx < cols || ldy < cols || !(eps >= 0.0f)) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype), wsize = twa_dtype_size(w_dtype);
  if (twa_misaligned_to(x, size) || twa_misaligned_to(y, size) || twa_misaligned_to(w, wsize) || twa_misaligned_to(b, wsize) ||
      twa_misaligned_to(mean, 4) || twa_misaligned_to(rstd, 4))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LnArgs a = {x, nullptr, y, w, b, mean, rstd, nullptr, ldx, 0, ldy, rows, cols, w_dtype, eps};
  const bool packs = ln_packs(x, ldx, cols, size) && ln_packs(y, ldy, cols, size);
  const LnPlan p = dtype == TWA_BF16 ? ln_plan<bf16, false>(ctx, packs, rows, cols) : ln_plan<float, false>(ctx, packs, rows, cols);
  if (p.kernel) {
    p.kernel<<<p.blocks, p.threads, p.smem, ctx->stream>>>(a);
  } else {
    const int blocks = static_cast<int>(rows < 8LL * ctx->sm_count ? rows : 8LL * ctx->sm_count);
    if (dtype == TWA_BF16) ln_forward_loop_kernel<bf16><<<blocks, LN_LOOP_THREADS, 0, ctx->stream>>>(a);
    else ln_forward_loop_kernel<float><<<blocks, LN_LOOP_THREADS, 0, ctx->stream>>>(a);
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

int twa_layer_norm_backward(twa_ctx* ctx, const void* dy, int64_t lddy, const void* x, int64_t ldx, twa_dtype dtype,
                            const void* w, twa_dtype w_dtype, const float* mean, const float* rstd, int64_t rows, int cols,
                            void* dx, int64_t lddx, void* dw, void* db, twa_dtype g_dtype, int accumulate, void* ws,
                            size_t ws_bytes) {
  int rc = ln_check(ctx, dtype, w_dtype, rows, cols);
  if (rc) return rc;
  if (!twa_dtype_ok(g_dtype) || accumulate < 0 || accumulate > 1) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (rows && (!dy || !x || !mean || !rstd || !dx || lddy < cols || ldx < cols || lddx < cols)) return TWA_ERR_INVALID_ARG;
  if (twa_misaligned_to(dy, size) || twa_misaligned_to(x, size) || twa_misaligned_to(dx, size) ||
      twa_misaligned_to(w, twa_dtype_size(w_dtype)) || twa_misaligned_to(mean, 4) || twa_misaligned_to(rstd, 4) ||
      twa_misaligned_to(dw, twa_dtype_size(g_dtype)) || twa_misaligned_to(db, twa_dtype_size(g_dtype)))
    return TWA_ERR_MISALIGNED;
  const bool weights = dw || db;
  if (weights) {
    if (!ws || ws_bytes < twa_layer_norm_workspace_bytes(rows, cols)) return TWA_ERR_WORKSPACE;
    if (twa_misaligned_to(ws, 16)) return TWA_ERR_MISALIGNED;
  }
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LnArgs a = {x, dy, dx, w, nullptr, const_cast<float*>(mean), const_cast<float*>(rstd),
              weights ? static_cast<float*>(ws) : nullptr, ldx, lddy, lddx, rows, cols, w_dtype, 0.0f};
  int parts = 0;
  if (rows) {
    const bool packs = ln_packs(x, ldx, cols, size) && ln_packs(dy, lddy, cols, size) && ln_packs(dx, lddx, cols, size);
    const LnPlan p = dtype == TWA_BF16 ? ln_plan<bf16, true>(ctx, packs, rows, cols) : ln_plan<float, true>(ctx, packs, rows, cols);
    if (p.kernel) {
      parts = p.blocks;
      p.kernel<<<p.blocks, p.threads, p.smem, ctx->stream>>>(a);
    } else {
      const int blocks = static_cast<int>(rows < 8LL * ctx->sm_count ? rows : 8LL * ctx->sm_count);
      if (weights) {
        parts = static_cast<int>(rows < 64 ? rows : 64);
        const dim3 grid(static_cast<unsigned>(twa_ceil_div(cols, 256)), parts);
        if (dtype == TWA_BF16) ln_weights_loop_kernel<bf16><<<grid, 256, 0, ctx->stream>>>(a);
        else ln_weights_loop_kernel<float><<<grid, 256, 0, ctx->stream>>>(a);
        TWA_CUDA_OK(ctx, cudaGetLastError());
      }
      if (dtype == TWA_BF16) ln_backward_loop_kernel<bf16><<<blocks, LN_LOOP_THREADS, 0, ctx->stream>>>(a);
      else ln_backward_loop_kernel<float><<<blocks, LN_LOOP_THREADS, 0, ctx->stream>>>(a);
    }
    TWA_CUDA_OK(ctx, cudaGetLastError());
  }
  if (weights) {
    ln_sum_kernel<<<static_cast<unsigned>(twa_ceil_div(2LL * cols, 32)), 32 * LN_SUM_WARPS, 0, ctx->stream>>>(
        static_cast<const float*>(ws), parts, cols, dw, db, g_dtype, accumulate);
    TWA_CUDA_OK(ctx, cudaGetLastError());
  }
  return TWA_OK;
}

}  // extern "C"
