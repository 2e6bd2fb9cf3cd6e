// Layer norm of rows and its gradient.
//
//   forward    mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps),
//              y = (x - mean) rstd w + b
//   backward   h = (x - mean) rstd,  v = dy w,
//              dx = rstd (v - sum v / cols - h sum(v h) / cols),   dw = sum_rows dy h,   db = sum_rows dy
//
// Both are bound by memory: a pass over x (and dy) and one store.  A row stays in the registers of the threads that
// share it, so it is read once, and the variance is taken from differences to a mean: a sum of squares would lose the
// digits that a mean far from zero costs.  Instructions come next: what a row costs beside its elements (the reductions, the
// root, addresses) is paid by every warp that shares it, so few threads share a row and hold many elements each, and sums
// and products go in pairs (16384 x 2048 bfloat16 with 8 elements a thread: 35 instructions an element, 45 us).
// Forward up to 2048 columns bfloat16 or 1024 float32 (backward 512) a warp or a part of one has a row and there is no
// barrier; above, a block has, with one barrier a row: forward each warp takes its own mean and the squares about it, and
// those combine exactly.
// The weights lie in shared memory as float32, whatever their type and alignment.  Backward a thread keeps the same
// columns for all its rows, and with them the columns' partial sums of dw and db in registers (from 8193 columns on in
// shared memory).  The partial sums of the blocks are added in float64 by a second kernel in block order, so results
// repeat bit for bit.
//
// 16384 x 2048 bfloat16: 25.7 us forward (134 MB, 5.2 TB/s), 40.5 us backward (201 MB, 5.0 TB/s), of which the sum of the
// blocks' parts takes 5; 4099 x 1023 float32 on no 16-byte boundary 17.8 us backward (50 MB): 7 rows a block, bound by the latency
// of a row and of the second launch.  16384 x 1023 bfloat16 on none 49 us backward (floor 15: every unit carries the tests of a
// row's ends, and only the next row is under way); 2048 x 12000 bfloat16 68 us (floor 22: one block an SM, no row under way).
#include "twa_layer_norm.cuh"

namespace {

// NV units a thread; FULL: the row is exactly the units of its threads, on 16-byte boundaries.
template <typename T, int E, int NV, int PER, bool FULL>
__global__ void __launch_bounds__(LN_THREADS<PER>, 512 / LN_THREADS<PER>) ln_forward_kernel(LnArgs a) {
  twa_begin(a.x, a.w, a.b);
  __shared__ float red[2][32][2];
  __shared__ float columns[32];                        // of each warp
  typedef LnPairs<E, NV> Q;
  constexpr int P = Q::P;
  int turn = 0;
  constexpr bool WARP = PER <= 32, ALONE = PER != 0;   // ALONE: a warp's threads are all of one row
  const LnPlace<E, NV, PER, FULL> at(a, sizeof(T));
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  const int units = at.units();
  const LnPlane<E> w = {0, units}, b = {units * E, units};
  const float inv = 1.0f / static_cast<float>(a.cols);
  twa_pack<T, E> raw[NV];
  auto fetch = [&](long long r) {
    if (r >= a.rows) return;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at.in(k)) at.load(raw[k], x + r * a.ldx, k, r > 0 && r + 1 < a.rows);
  };
  fetch(at.first + at.group);
  ln_stage<E>(w, a.w, a.w_dtype, at.skew, a.cols, 1.0f);
  ln_stage<E>(b, a.b, a.w_dtype, at.skew, a.cols, 0.0f);
  float inv_warp = 0.0f;
  if (!WARP) {
    int mine = 0;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) mine += at.valid(k, e) ? 1 : 0;
    const float n = twa_warp_sum(static_cast<float>(mine));
    inv_warp = n > 0.0f ? 1.0f / n : 0.0f;
    if ((threadIdx.x & 31) == 0) columns[threadIdx.x >> 5] = n;
  }
  __syncthreads();
  for (long long base = at.first; base < a.rows; base += at.step) {
    const long long r = base + at.group;
    float f[Q::N];
    twa_f2 v[P], s2 = 0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if ((!ALONE && r >= a.rows) || !at.in(k)) raw[k] = twa_pack<T, E>{};
      raw[k].widen(f + k * E);
      at.keep_valid(k, f + k * E);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      v[i] = Q::get(f, i);
      s2 = twa_add2(s2, v[i]);
    }
    // the mean of the row, or of the warp's columns, and the squares about it
    const float s = WARP ? ln_sum_lanes<PER>(twa_pair_sum(s2), a.log_lanes) : twa_warp_sum(twa_pair_sum(s2));
    float mean = s * (WARP ? inv : inv_warp);
    const twa_f2 m2 = twa_pair(-mean);
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = twa_add2(v[i], m2);        // differences to this mean from here on
    if (!FULL) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (!at.whole(k))
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (!at.valid(k, e)) {
              const int i = (k * E + e) / 2;
              float lo, hi;
              twa_unpair(v[i], lo, hi);
              v[i] = (k * E + e) % 2 ? twa_pair(lo, 0.0f) : twa_pair(0.0f, hi);
            }
    }
    twa_f2 q2 = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) q2 = twa_fma2(v[i], v[i], q2);
    if (Q::N == 1) q2 = twa_mul2(q2, twa_pair(1.0f, 0.0f));       // a pair of one element
    float q = WARP ? ln_sum_lanes<PER>(twa_pair_sum(q2), a.log_lanes) : twa_warp_sum(twa_pair_sum(q2));
    if (!WARP) {
      // squares about the row's mean: those about the warps' means, and columns x (difference of the means)^2
      float(*set)[2] = red[turn];
      turn ^= 1;
      if ((threadIdx.x & 31) == 0) {
        set[threadIdx.x >> 5][0] = mean;
        set[threadIdx.x >> 5][1] = q;
      }
      __syncthreads();
      constexpr int warps = PER / 32;
      float all = 0.0f;
#pragma unroll
      for (int k = 0; k < warps; ++k) all += columns[k] * set[k][0];
      all *= inv;
      q = 0.0f;
#pragma unroll
      for (int k = 0; k < warps; ++k) {
        const float d = set[k][0] - all;
        q += set[k][1] + columns[k] * d * d;
      }
      const twa_f2 off = twa_pair(mean - all);
      mean = all;
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = twa_add2(v[i], off);
    }
    const float rstd = rsqrtf(q * inv + a.eps);
    fetch(r + at.step);
    if (ALONE || r < a.rows) {
      if (at.t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
      }
      const twa_f2 r2 = twa_pair(rstd);
#pragma unroll
      for (int i = 0; i < P; ++i) Q::put(f, i, twa_mul2(v[i], r2));
      T* row = y + r * a.ldy;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (at.in(k)) {
          float wv[E], bv[E], o[E];
          w.load(at.unit(k), wv);
          b.load(at.unit(k), bv);
          if constexpr (E == 1) {
            o[0] = fmaf(f[k], wv[0], bv[0]);
          } else {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              const twa_f2 p = twa_fma2(twa_pair(f[k * E + e], f[k * E + e + 1]), twa_pair(wv[e], wv[e + 1]), twa_pair(bv[e], bv[e + 1]));
              twa_unpair(p, o[e], o[e + 1]);
            }
          }
          at.store(row, k, o);
        }
    }
  }
}

// Rows of any width, a block per row: the row is read again for each of its passes (from L2, while it fits there).
template <typename T>
__global__ void ln_forward_loop_kernel(LnArgs a) {
  twa_begin(a.x, a.w, a.b);
  __shared__ float red[2][32][2];
  int turn = 0;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* xr = x + r * a.ldx;
    float s[2] = {0.0f, 0.0f};
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) s[0] += twa_to_float(xr[c]);
    ln_block_sums<0>(s, red, turn);
    const float mean = s[0] / static_cast<float>(a.cols);
    float q[2] = {0.0f, 0.0f};
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float d = twa_to_float(xr[c]) - mean;
      q[0] += d * d;
    }
    ln_block_sums<0>(q, red, turn);
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

struct LnForward {
  template <int E, int PER>
  static constexpr int HELD = PER == 32 && E == 8 ? 64 : 32;
  static constexpr long long MAX_BLOCKS = 1LL << 30;
  static size_t ring_bytes(int, int, bool) { return 0; }
  template <typename T, int E, int NV, int PER>
  static LnKernel kernel(bool aligned, bool full) {
    if constexpr (E > 1 && PER > 0)
      if (aligned && full) return ln_forward_kernel<T, E, NV, PER, true>;
    return ln_forward_kernel<T, E, NV, PER, false>;
  }
  template <typename T, int E>
  static void wide(int, LnPlan*) {}
};

}  // namespace

extern "C" {

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
  LnArgs a = {x, nullptr, y, w, b, mean, rstd, nullptr, ldx, 0, ldy, rows, cols, w_dtype, 5, 0, eps, ctx->wait_limit_ns, ctx->d_status};
  const int classes = ln_classes(x, ldx, y, ldy, y, ldy, rows, cols, size);
  LnPlan p;
  rc = dtype == TWA_BF16 ? ln_plan<LnForward, bf16>(ctx, classes, rows, cols, &p) : ln_plan<LnForward, float>(ctx, classes, rows, cols, &p);
  if (rc) return rc;
  a.log_lanes = p.log_lanes;
  a.log_classes = p.log_classes;
  if (p.kernel) {
    twa_launch(ctx->stream, p.kernel, p.blocks, p.threads, p.smem, a);
  } else {
    const int blocks = static_cast<int>(rows < 8LL * ctx->sm_count ? rows : 8LL * ctx->sm_count);
    if (dtype == TWA_BF16) twa_launch(ctx->stream, ln_forward_loop_kernel<bf16>, blocks, LN_LOOP_THREADS, 0, a);
    else twa_launch(ctx->stream, ln_forward_loop_kernel<float>, blocks, LN_LOOP_THREADS, 0, a);
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
