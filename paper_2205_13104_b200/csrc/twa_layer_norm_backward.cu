// Gradient of layer norm: dx, dw and db (formulas and design beside the forward pass, twa_layer_norm.cu).
#include "twa_layer_norm.cuh"

namespace {

// NV units a thread.  RING (rows on 16-byte boundaries, a warp or a block each): LN_RING_ROWS rows of x and dy are under way as bulk
// copies into shared memory, which costs no registers; else the next row is on its way into registers.  FULL: as forward.
template <int NV>
constexpr int LN_RING_ROWS = NV >= 3 ? 2 : 4;      // 16 KB of x and dy a block of 128 threads either way, four blocks an SM
template <typename T, int E, int NV, int PER, bool FULL, bool RING>
__global__ void __launch_bounds__(LN_THREADS<PER>, 512 / LN_THREADS<PER>) ln_backward_kernel(LnArgs a) {
  constexpr bool WARP = PER <= 32, ALONE = PER != 0;   // ALONE: a warp's threads are all of one row
  constexpr int LN_RING = LN_RING_ROWS<NV>;
  constexpr int TEAMS = PER == 32 ? LN_WARP_THREADS / 32 : 1, ROW = PER * NV;      // rings of a block, units of a row in one
  __shared__ __align__(16) float red[2][32][2];
  __shared__ unsigned long long full[RING ? TEAMS * LN_RING : 1];
  __shared__ int gave_up;
  typedef LnPairs<E, NV> Q;
  constexpr int P = Q::P;
  int turn = 0;
  const LnPlace<E, NV, PER, FULL> at(a, sizeof(T));
  const LnPlane<E> w = {0, at.units()};
  const int team = PER == 32 ? threadIdx.x >> 5 : 0;
  const bool issuer = RING && (PER == 32 ? (threadIdx.x & 31) == 0 : threadIdx.x == 0);
  uint4* ring = reinterpret_cast<uint4*>(ln_planes + 2 * at.units() * E) + team * LN_RING * 2 * ROW;
  if (RING) {
    if (threadIdx.x == 0) {
      for (int q = 0; q < TEAMS * LN_RING; ++q) twa_mbar_init(twa_smem_u32(&full[q]), 1);
      gave_up = 0;
      twa_fence_barrier_init();
    }
    __syncthreads();
  }
  twa_begin(a.x, a.dy, a.w, a.mean, a.rstd);
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.y);
  const float inv = 1.0f / static_cast<float>(a.cols);
  twa_f2 dw[P], db[P];
#pragma unroll
  for (int i = 0; i < P; ++i) dw[i] = db[i] = 0;
  twa_pack<T, E> rx[NV] = {}, rd[NV] = {};             // what is beyond the row stays 0 in rd, and with it all that is added up
  float mean = 0.0f, rstd = 0.0f;
  // copies of the team's i-th row, where there is one
  auto issue = [&](int i) {
    const long long r = at.first + i * at.step;
    if (r >= a.rows) return;
    const int q = i % LN_RING;
    const uint32_t bytes = (FULL ? ROW : at.row_units) * 16;
    unsigned long long* bar = &full[team * LN_RING + q];
    twa_mbar_expect_tx(twa_smem_u32(bar), 2 * bytes);
    twa_bulk_load(twa_smem_u32(ring + q * 2 * ROW), x + r * a.ldx, bytes, twa_smem_u32(bar));
    twa_bulk_load(twa_smem_u32(ring + q * 2 * ROW + ROW), dy + r * a.lddy, bytes, twa_smem_u32(bar));
  };
  auto fetch = [&](long long r) {
    if (r >= a.rows) return;
    mean = __ldg(a.mean + r);
    rstd = __ldg(a.rstd + r);
    if (!RING)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (at.in(k)) {
          const bool inner = r > 0 && r + 1 < a.rows;
          at.load(rx[k], x + r * a.ldx, k, inner);
          at.load(rd[k], dy + r * a.lddy, k, inner);
        }
  };
  if (issuer)
    for (int i = 0; i < LN_RING; ++i) issue(i);
  fetch(at.first + at.group);
  ln_stage<E>(w, a.w, a.w_dtype, at.skew, a.cols, 1.0f);
  __syncthreads();
  int it = 0;
  bool landed = true;
  for (long long base = at.first; base < a.rows; base += at.step, ++it) {
    const long long r = base + at.group;
    twa_f2 h[P], v[P], s0 = 0, s1 = 0;
    const float rs = rstd;
    if constexpr (RING) {
      const int q = it % LN_RING;
      if (!twa_wait(&full[team * LN_RING + q], it / LN_RING & 1, &gave_up, a.wait_limit_ns)) {
        // The results are not defined, and every later wait ends at once.  Nothing is copied any more: the last copy into the
        // place of a row may not have landed; and none may still be on its way into this block's shared memory when it ends.
        if (issuer && landed)
          for (int i = it; i < it + LN_RING && at.first + i * at.step < a.rows; ++i) {
            const unsigned long long begun = twa_globaltimer();
            while (!twa_mbar_try_wait(twa_smem_u32(&full[team * LN_RING + i % LN_RING]), i / LN_RING & 1))
              if (twa_globaltimer() - begun > a.wait_limit_ns) break;
          }
        landed = false;
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (at.in(k)) {
          rx[k].load_shared(ring + q * 2 * ROW + at.unit(k));
          rd[k].load_shared(ring + q * 2 * ROW + ROW + at.unit(k));
        }
    }
    if (ALONE || r < a.rows) {
      float f[Q::N], d[Q::N], wv[Q::N];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        rx[k].widen(f + k * E);
        rd[k].widen(d + k * E);
        if (!RING) {
          at.keep_valid(k, f + k * E);
          at.keep_valid(k, d + k * E);
        }
        w.load(at.unit(k), wv + k * E);
      }
      const twa_f2 m2 = twa_pair(-mean), r2 = twa_pair(rs);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const twa_f2 di = Q::get(d, i);
        h[i] = twa_mul2(twa_add2(Q::get(f, i), m2), r2);
        dw[i] = twa_fma2(di, h[i], dw[i]);
        db[i] = twa_add2(db[i], di);
        v[i] = twa_mul2(di, Q::get(wv, i));
        s0 = twa_add2(s0, v[i]);
        s1 = twa_fma2(v[i], h[i], s1);
      }
    }
    fetch(r + at.step);
    float s[2] = {twa_pair_sum(s0), twa_pair_sum(s1)};
    if constexpr (PER == 32) {
      const float mine = ln_two_sums(s[0], s[1]), other = __shfl_xor_sync(0xffffffffu, mine, 16);
      s[0] = threadIdx.x & 16 ? other : mine;
      s[1] = threadIdx.x & 16 ? mine : other;
    } else if constexpr (WARP) {
      s[0] = ln_sum_lanes<PER>(s[0], a.log_lanes);
      s[1] = ln_sum_lanes<PER>(s[1], a.log_lanes);
    } else {
      ln_block_sums<PER / 32>(s, red, turn);           // and with its barrier the row has been read
    }
    if (WARP) __syncwarp();
    if (issuer && landed) issue(it + LN_RING);
    if (ALONE || r < a.rows) {
      // rstd (v - c1 - h c2)
      const twa_f2 c1 = twa_pair(-s[0] * inv), c2 = twa_pair(-s[1] * inv), r2 = twa_pair(rs);
      float f[Q::N];
#pragma unroll
      for (int i = 0; i < P; ++i) Q::put(f, i, twa_mul2(r2, twa_fma2(h[i], c2, twa_add2(v[i], c1))));
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (at.in(k)) at.store(dx + r * a.ldy, k, f + k * E);
    }
  }
  if (RING && !landed) twa_set_status(a.status, TWA_ERR_TIMEOUT, -1);
  if (!a.part) return;
  float* out = a.part + static_cast<long long>(blockIdx.x) * 2 * a.cols;
  if constexpr (WARP) {
    // the rows of a warp side by side
#pragma unroll
    for (int i = 0; i < P; ++i)
      for (int o = PER ? 5 : a.log_lanes; o < 5; ++o) {
        dw[i] = twa_add2(dw[i], __shfl_xor_sync(0xffffffffu, dw[i], 1 << o));
        db[i] = twa_add2(db[i], __shfl_xor_sync(0xffffffffu, db[i], 1 << o));
      }
  }
  float fw[Q::N], fb[Q::N];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    Q::put(fw, i, dw[i]);
    Q::put(fb, i, db[i]);
  }
  if constexpr (WARP) {
    for (int which = 0; which < LN_WARP_THREADS / 32; ++which) {      // the warps in order
      __syncthreads();
      if (which == static_cast<int>(threadIdx.x >> 5) && at.group == 0)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (at.valid(k, e)) {
              const int c = at.column(k, e);
              ln_planes[c] = which ? ln_planes[c] + fw[k * E + e] : fw[k * E + e];
              ln_planes[a.cols + c] = which ? ln_planes[a.cols + c] + fb[k * E + e] : fb[k * E + e];
            }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.cols; c += blockDim.x) out[c] = ln_planes[c];
  } else if constexpr (FULL) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        twa_pack<float, 4>::store(out + at.column(k, e), fw + k * E + e);
        twa_pack<float, 4>::store(out + a.cols + at.column(k, e), fb + k * E + e);
      }
  } else {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (at.valid(k, e)) {
          out[at.column(k, e)] = fw[k * E + e];
          out[a.cols + at.column(k, e)] = fb[k * E + e];
        }
  }
}

// Rows of 8193 .. 16384 columns: a block of 1024 threads, 16 elements a thread as they lie in memory, the weights and the partial
// sums of dw and db in shared memory.
template <typename T, int E>
__global__ void __launch_bounds__(LN_WIDE_THREADS) ln_backward_wide_kernel(LnArgs a) {
  twa_begin(a.x, a.dy, a.w, a.mean, a.rstd);
  __shared__ __align__(16) float red[2][32][2];
  int turn = 0;
  constexpr int NV = LN_WIDE_HELD / E;
  const int units = (a.cols + E - 1) / E, t = threadIdx.x;
  const LnPlane<E> w = {0, units}, dw = {units * E, units}, db = {2 * units * E, units};
  ln_stage<E>(w, a.w, a.w_dtype, 0, a.cols, 1.0f);
  for (int c = t; c < 2 * units * E; c += LN_WIDE_THREADS) ln_planes[units * E + c] = 0.0f;
  __syncthreads();
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.y);
  const float inv = 1.0f / static_cast<float>(a.cols);
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float mean = __ldg(a.mean + r), rstd = __ldg(a.rstd + r);
    twa_pack<T, E> rx[NV], rd[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (k * LN_WIDE_THREADS + t < units) {
        rx[k].load(x + r * a.ldx + (k * LN_WIDE_THREADS + t) * E);
        rd[k].load(dy + r * a.lddy + (k * LN_WIDE_THREADS + t) * E);
      }
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int u = k * LN_WIDE_THREADS + t;
      if (u >= units) continue;
      float h[E], d[E], q[E];
      rx[k].widen(h);
      rd[k].widen(d);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = (h[e] - mean) * rstd;
      dw.load(u, q);
#pragma unroll
      for (int e = 0; e < E; ++e) q[e] += d[e] * h[e];
      dw.store(u, q);
      db.load(u, q);
#pragma unroll
      for (int e = 0; e < E; ++e) q[e] += d[e];
      db.store(u, q);
      w.load(u, q);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = d[e] * q[e];
        s[0] += v;
        s[1] += v * h[e];
      }
    }
    ln_block_sums<0>(s, red, turn);
    const float c1 = s[0] * inv, c2 = s[1] * inv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int u = k * LN_WIDE_THREADS + t;
      if (u >= units) continue;
      float h[E], d[E], q[E];
      rx[k].widen(h);
      rd[k].widen(d);
      w.load(u, q);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = rstd * (d[e] * q[e] - c1 - (h[e] - mean) * rstd * c2);
      twa_pack<T, E>::store(dx + r * a.ldy + u * E, h);
    }
  }
  if (!a.part) return;
  float* out = a.part + static_cast<long long>(blockIdx.x) * 2 * a.cols;
  __syncthreads();
  for (int c = t; c < a.cols; c += LN_WIDE_THREADS) {
    out[c] = ln_planes[dw.at(c / E, c % E)];
    out[a.cols + c] = ln_planes[db.at(c / E, c % E)];
  }
}

template <typename T>
__global__ void ln_backward_loop_kernel(LnArgs a) {
  twa_begin(a.x, a.dy, a.w, a.b, a.mean, a.rstd);
  __shared__ __align__(16) float red[2][32][2];
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
    ln_block_sums<0>(s, red, turn);
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
__global__ void ln_weights_loop_kernel(LnArgs a) {
  twa_begin(a.x, a.dy, a.w, a.b, a.mean, a.rstd);
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

// Adds the blocks' partial sums: 32 columns a block, a warp for every LN_SUM_WARPS-th of the blocks' rows, all loads of a thread
// under way at once; then a warp a column, in a fixed tree.
constexpr int LN_SUM_WARPS = 32, LN_SUM_EACH = (LN_MAX_BLOCKS + LN_SUM_WARPS - 1) / LN_SUM_WARPS;
__global__ void __launch_bounds__(32 * LN_SUM_WARPS) ln_sum_kernel(const float* part, int blocks, int cols, void* dw, void* db,
                                                                  int g_dtype, int accumulate) {
  twa_begin(part, dw, db);
  __shared__ double run[LN_SUM_WARPS][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int c = blockIdx.x * 32 + lane;                     // 0 .. 2 cols - 1: dw, then db
  float v[LN_SUM_EACH];
#pragma unroll
  for (int k = 0; k < LN_SUM_EACH; ++k) {
    const int b = k * LN_SUM_WARPS + warp;
    v[k] = b < blocks && c < 2 * cols ? __ldg(part + static_cast<long long>(b) * 2 * cols + c) : 0.0f;
  }
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < LN_SUM_EACH; ++k) s += static_cast<double>(v[k]);
  run[warp][lane] = s;
  __syncthreads();
  c = blockIdx.x * 32 + warp;
  s = run[lane][warp];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane || c >= 2 * cols) return;
  void* out = c < cols ? dw : db;
  const int i = c < cols ? c : c - cols;
  if (!out) return;
  if (accumulate) s += static_cast<double>(twa_load_any(out, g_dtype, i));
  twa_store_any(out, g_dtype, i, static_cast<float>(s));
}

// x, dy and two sums a column take the registers.
struct LnBackward {
  template <int E, int PER>
  static constexpr int HELD = 16;
  static constexpr long long MAX_BLOCKS = LN_MAX_BLOCKS;
  static size_t ring_bytes(int per, int nv, bool aligned) {
    if (!aligned || per < 32) return 0;
    return 16LL * 2 * per * nv * (nv >= 3 ? LN_RING_ROWS<3> : LN_RING_ROWS<1>) * (per == 32 ? LN_WARP_THREADS / 32 : 1);
  }
  template <typename T, int E, int NV, int PER>
  static LnKernel kernel(bool aligned, bool full) {
    if constexpr (E > 1 && PER > 0) {
      if (aligned && full) return ln_backward_kernel<T, E, NV, PER, true, true>;
      if (aligned) return ln_backward_kernel<T, E, NV, PER, false, true>;
    }
    return ln_backward_kernel<T, E, NV, PER, false, false>;
  }
  template <typename T, int E>
  static void wide(int units, LnPlan* p) {
    if (units > LN_WIDE_THREADS * (LN_WIDE_HELD / E)) return;
    p->threads = LN_WIDE_THREADS;
    p->smem = sizeof(float) * 3 * units * E;
    p->kernel = ln_backward_wide_kernel<T, E>;
  }
};

}  // namespace

extern "C" {

size_t twa_layer_norm_workspace_bytes(int64_t rows, int cols) {
  if (rows < 0 || cols < 1) return 0;
  const long long most = cols > LN_WIDE_THREADS * LN_WIDE_HELD ? LN_LOOP_PARTS : LN_MAX_BLOCKS;
  const long long blocks = rows < most ? (rows + 8) / 8 * 8 : most;      // a plan rounds up by classes
  return twa_round256(sizeof(float) * 2 * static_cast<size_t>(cols) * blocks);
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
  if (rows && (twa_misaligned_to(dy, size) || twa_misaligned_to(x, size) || twa_misaligned_to(dx, size) ||
               twa_misaligned_to(mean, 4) || twa_misaligned_to(rstd, 4)))
    return TWA_ERR_MISALIGNED;
  if (twa_misaligned_to(w, twa_dtype_size(w_dtype)) || twa_misaligned_to(dw, twa_dtype_size(g_dtype)) ||
      twa_misaligned_to(db, twa_dtype_size(g_dtype)))
    return TWA_ERR_MISALIGNED;
  const bool weights = dw || db;
  if (weights) {
    if (!ws || ws_bytes < twa_layer_norm_workspace_bytes(rows, cols)) return TWA_ERR_WORKSPACE;
    if (twa_misaligned_to(ws, 16)) return TWA_ERR_MISALIGNED;
  }
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LnArgs a = {x, dy, dx, w, nullptr, const_cast<float*>(mean), const_cast<float*>(rstd),
              weights ? static_cast<float*>(ws) : nullptr, ldx, lddy, lddx, rows, cols, w_dtype, 5, 0, 0.0f, ctx->wait_limit_ns, ctx->d_status};
  int parts = 0;
  if (rows) {
    const int classes = ln_classes(x, ldx, dy, lddy, dx, lddx, rows, cols, size);
    LnPlan p;
    rc = dtype == TWA_BF16 ? ln_plan<LnBackward, bf16>(ctx, classes, rows, cols, &p) : ln_plan<LnBackward, float>(ctx, classes, rows, cols, &p);
    if (rc) return rc;
    a.log_lanes = p.log_lanes;
    a.log_classes = p.log_classes;
    if (p.kernel) {
      parts = p.blocks;
      twa_launch(ctx->stream, p.kernel, p.blocks, p.threads, p.smem, a);
    } else {
      const int blocks = static_cast<int>(rows < 8LL * ctx->sm_count ? rows : 8LL * ctx->sm_count);
      if (weights) {
        parts = static_cast<int>(rows < LN_LOOP_PARTS ? rows : LN_LOOP_PARTS);
        const dim3 grid(static_cast<unsigned>(twa_ceil_div(cols, 256)), parts);
        if (dtype == TWA_BF16) twa_launch(ctx->stream, ln_weights_loop_kernel<bf16>, grid, 256, 0, a);
        else twa_launch(ctx->stream, ln_weights_loop_kernel<float>, grid, 256, 0, a);
        TWA_CUDA_OK(ctx, cudaGetLastError());
      }
      if (dtype == TWA_BF16) twa_launch(ctx->stream, ln_backward_loop_kernel<bf16>, blocks, LN_LOOP_THREADS, 0, a);
      else twa_launch(ctx->stream, ln_backward_loop_kernel<float>, blocks, LN_LOOP_THREADS, 0, a);
    }
    TWA_CUDA_OK(ctx, cudaGetLastError());
  }
  if (weights) {
    twa_launch(ctx->stream, ln_sum_kernel, static_cast<unsigned>(twa_ceil_div(2LL * cols, 32)), 32 * LN_SUM_WARPS, 0, static_cast<const float*>(ws), parts, cols, dw, db, g_dtype, accumulate);
    TWA_CUDA_OK(ctx, cudaGetLastError());
  }
  return TWA_OK;
}

}  // extern "C"
