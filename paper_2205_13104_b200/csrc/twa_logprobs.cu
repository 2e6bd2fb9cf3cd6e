// Log probabilities of given tokens with the entropy of their distribution and its most likely tokens, and the
// gradient of both.  For a row z of logits, p = softmax(z):
//
//   forward    lse = log sum exp z,  logp = z[target] - lse,  H = lse - sum p z = log S - A / S
//              with m = max z, S = sum exp(z - m), A = sum exp(z - m) (z - m)
//   backward   dz[j] = d_logp ([j == target] - p[j]) - d_H p[j] (log p[j] + H)
//
// Forward is one pass: every thread keeps the running m, S and A of the elements it meets (S and A are rescaled when m
// grows); the threads' triples are merged at the end.  Exponents are differences to the maximum times log2 e: a mask of
// the type's lowest value would overflow if the product came first, and far from zero the difference is the more exact.
// Backward is one read and one write.  Both are bound by memory.
//
// The most likely tokens cost no second pass.  Each thread also remembers in which 16-byte unit of its elements its
// maximum lay.  Order all elements by (value, smaller unit first): the k-th best of the threads' maxima, T, bounds the
// k-th best element from below, because the k maxima are k elements; so every one of the k best elements ranks at or
// above T, and lies in one of the k threads whose maximum does.  Only those threads look at their elements again (in
// L2), and the few elements that rank at or above T are sorted by (value, smaller index first).
#include "twa_ops.cuh"

namespace {

constexpr int LP_THREADS = 512, LP_WARPS = LP_THREADS / 32;
constexpr int LP_MAX_CLUSTER = 8;
constexpr int LP_BUFFER = LP_THREADS;           // candidates that are sorted at once
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
typedef unsigned long long u64;

__device__ __forceinline__ float lp_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Order-preserving bits of a value; zeros of both signs are equal.  0 is below every value, -inf included.
__device__ __forceinline__ uint32_t lp_rank(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float lp_unrank(uint32_t r) {
  return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r);
}
__device__ __forceinline__ u64 lp_key(float v, uint32_t place) { return static_cast<u64>(lp_rank(v)) << 32 | (0xffffffffu - place); }

// A row as 16-byte units counted from the aligned address at or below its first element; the first and the last
// unit may be partly outside and are read element by element.
template <typename T>
struct LpRow {
  static constexpr int E = twa_vec<T>;
  const T* base;       // unit 0, element 0 (may lie before the row)
  int skew, cols;      // the row's element j is base[skew + j]
  __device__ __forceinline__ LpRow(const T* row, int n) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row);
    skew = static_cast<int>((a & 15) / sizeof(T));
    base = reinterpret_cast<const T*>(a & ~static_cast<uintptr_t>(15));
    cols = n;
  }
  __device__ __forceinline__ int units() const { return (skew + cols + E - 1) / E; }
  __device__ __forceinline__ bool whole(int u) const { return u * E >= skew && (u + 1) * E <= skew + cols; }
  // Elements outside the row are -inf, and `valid` has their bits clear.
  __device__ __forceinline__ unsigned load_partial(int u, float* v) const {
    unsigned valid = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = u * E + e - skew;
      const bool in = j >= 0 && j < cols;
      v[e] = in ? twa_to_float(base[u * E + e]) : -INFINITY;
      valid |= in ? 1u << e : 0u;
    }
    return valid;
  }
};

// Sums of some elements of a row: m = their maximum (-inf: none above -inf), with d = (z - m) log2 e
// s = sum 2^d, a = sum 2^d d.
struct LpStat {
  float m, s, a;
};
template <bool ENT>
__device__ __forceinline__ LpStat lp_merge(const LpStat& x, const LpStat& y) {
  LpStat r;
  r.m = fmaxf(x.m, y.m);
  const float base = r.m == -INFINITY ? 0.0f : r.m;
  // a side without any value (m = -inf) has the sums 0, or NaN where a NaN was met
  const float dx = fmaxf((x.m - base) * LOG2E, -150.0f), dy = fmaxf((y.m - base) * LOG2E, -150.0f);
  const float fx = lp_exp2(dx), fy = lp_exp2(dy);
  r.s = x.s * fx + y.s * fy;
  r.a = ENT ? fx * (x.a + dx * x.s) + fy * (y.a + dy * y.s) : 0.0f;
  return r;
}

// ---- the best 32 of a block's keys -------------------------------------------------------------------
__device__ __forceinline__ u64 lp_shfl_xor(u64 v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }

// Sorts 32 keys of a warp, largest in lane 0 (bitonic network).
__device__ __forceinline__ u64 lp_sort32(u64 v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j; j >>= 1) {
      const u64 o = lp_shfl_xor(v, j);
      const bool keep_max = ((lane & j) == 0) == ((lane & k) == 0 || k == 32);
      v = keep_max ? (v > o ? v : o) : (v < o ? v : o);
    }
  return v;
}
// The 32 best of two sorted lists, sorted: `other` is lane's entry of the second list reversed.
__device__ __forceinline__ u64 lp_merge32(u64 v, u64 other_reversed) {
  const int lane = threadIdx.x & 31;
  v = v > other_reversed ? v : other_reversed;
#pragma unroll
  for (int j = 16; j; j >>= 1) {
    const u64 o = lp_shfl_xor(v, j);
    v = (lane & j) == 0 ? (v > o ? v : o) : (v < o ? v : o);
  }
  return v;
}
// The block's 32 best of one key per thread, sorted, in the lanes of warp 0 (other warps: undefined).
__device__ __forceinline__ u64 lp_block_best(u64 v, u64 (*list)[32]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  v = lp_sort32(v);
  for (int half = LP_WARPS / 2; half; half >>= 1) {
    if (warp >= half && warp < 2 * half) list[warp][lane] = v;
    __syncthreads();
    if (warp < half) v = lp_merge32(v, list[warp + half][31 - lane]);
    __syncthreads();
  }
  return v;
}

struct LpArgs {
  const void* logits;
  const void* targets;
  float *logp, *lse, *entropy;
  int* top_ids;
  float* top_logp;
  const float *d_logp, *d_entropy;
  void* dlogits;
  long long ld, ldd, rows, ignore_id;
  int vocab, itype, top;
  int* status;
};

struct LpShared {
  u64 list[LP_WARPS][32];
  u64 buffer[LP_BUFFER];
  u64 best[32];                // this block's best, read by the first block of the cluster
  LpStat stat[LP_WARPS];
  LpStat mine;                 // this block's sums, read by the first block of the cluster
  u64 bound;
  int count;
  u64 round;
};

__device__ __forceinline__ uint32_t lp_cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void lp_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename V>
__device__ __forceinline__ V lp_remote(const V* p, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(twa_smem_u32(p)), "r"(rank));
  V v;
  if constexpr (sizeof(V) == 8) {
    u64 w;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(w) : "r"(at) : "memory");
    v = w;
  } else {
    uint32_t w;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
    memcpy(&v, &w, 4);
  }
  return v;
}

// A row per cluster of `parts` blocks; units are dealt to the cluster's threads in turn.
template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(const LpArgs a, const int parts) {
  constexpr int E = twa_vec<T>;
  __shared__ LpShared sh;
  const uint32_t part = parts > 1 ? lp_cluster_rank() : 0;
  const long long row = blockIdx.x / parts;
  const LpRow<T> x(static_cast<const T*>(a.logits) + row * a.ld, a.vocab);
  const int units = x.units(), stride = LP_THREADS * parts, first = static_cast<int>(part) * LP_THREADS + threadIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

  float m = -INFINITY, s = 0.0f, w = 0.0f;
  int best = first;
  auto take = [&](const float* v, int u) {
    float um = v[0];
#pragma unroll
    for (int e = 1; e < E; ++e) um = fmaxf(um, v[e]);
    if (um == -INFINITY) return;
    if (um > m) {
      if (m > -INFINITY) {
        const float d = fmaxf((m - um) * LOG2E, -150.0f), f = lp_exp2(d);
        if (ENT) w = f * (w + d * s);
        s *= f;
      }
      m = um;
      best = u;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = (v[e] - m) * LOG2E, p = lp_exp2(d);
      s += p;
      if (ENT) w = fmaf(p, fmaxf(d, -150.0f), w);
    }
  };
  constexpr int AHEAD = 4;
  for (int u0 = first; u0 < units; u0 += AHEAD * stride) {
    twa_pack<T, E> q[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int u = u0 + k * stride;
      if (u < units && x.whole(u)) q[k].load(x.base + static_cast<long long>(u) * E);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int u = u0 + k * stride;
      if (u >= units) break;
      float v[E];
      if (x.whole(u)) q[k].widen(v);
      else x.load_partial(u, v);
      take(v, u);
    }
  }

  // the block's sums
  LpStat st = {m, s, w};
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    LpStat other;
    other.m = __shfl_xor_sync(0xffffffffu, st.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, st.s, o);
    other.a = ENT ? __shfl_xor_sync(0xffffffffu, st.a, o) : 0.0f;
    st = lp_merge<ENT>(st, other);
  }
  if (lane == 0) sh.stat[warp] = st;
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
  if (warp == 0) {
    st = lane < LP_WARPS ? sh.stat[lane] : LpStat{-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int o = LP_WARPS / 2; o; o >>= 1) {
      LpStat other;
      other.m = __shfl_xor_sync(0xffffffffu, st.m, o);
      other.s = __shfl_xor_sync(0xffffffffu, st.s, o);
      other.a = ENT ? __shfl_xor_sync(0xffffffffu, st.a, o) : 0.0f;
      st = lp_merge<ENT>(st, other);
    }
    if (lane == 0) sh.mine = st;
  }

  u64 found = 0;                 // warp 0: the block's best, sorted
  if (TOP) {
    const u64 mine = first < units ? lp_key(m, best) : 0;
    const u64 heads = lp_block_best(mine, sh.list);
    if (warp == 0 && lane == a.top - 1) sh.bound = heads;
    __syncthreads();
    const u64 bound = sh.bound;
    auto scan = [&](auto&& use) {
      if (mine == 0 || mine < bound) return;
      for (int u = first; u < units; u += stride) {
        float v[E];
        unsigned valid = (1u << E) - 1;
        if (x.whole(u)) {
          twa_pack<T, E> q;
          q.load(x.base + static_cast<long long>(u) * E);
          q.widen(v);
        } else {
          valid = x.load_partial(u, v);
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
          if ((valid >> e & 1) && lp_key(v[e], u) >= bound) use(lp_key(v[e], u * E + e - x.skew));
      }
    };
    scan([&](u64 key) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < LP_BUFFER) sh.buffer[at] = key;
    });
    __syncthreads();
    if (sh.count <= LP_BUFFER) {
      found = lp_block_best(static_cast<int>(threadIdx.x) < sh.count ? sh.buffer[threadIdx.x] : 0, sh.list);
    } else {
      // too many elements rank with the bound (a row with many equal values): one round per token
      u64 below = ~0ull;
      for (int i = 0; i < a.top; ++i) {
        u64 top = 0;
        scan([&](u64 key) { if (key < below && key > top) top = key; });
        if (threadIdx.x == 0) sh.round = 0;
        __syncthreads();
        if (top) atomicMax(&sh.round, top);
        __syncthreads();
        below = sh.round;
        if (lane == i) found = below;
        __syncthreads();
      }
    }
    if (warp == 0) sh.best[lane] = found;
  }

  // the cluster's
  if (parts > 1) {
    lp_cluster_sync();
    if (part == 0 && warp == 0) {
      for (int p = 1; p < parts; ++p) {
        LpStat other;
        other.m = lp_remote(&sh.mine.m, p);
        other.s = lp_remote(&sh.mine.s, p);
        other.a = ENT ? lp_remote(&sh.mine.a, p) : 0.0f;
        if (lane == 0) st = lp_merge<ENT>(st, other);
        if (TOP) found = lp_merge32(found, lp_remote(&sh.best[31 - lane], p));
      }
    }
    lp_cluster_sync();           // no block leaves while its shared memory is read
  }
  if (part != 0 || warp != 0) return;
  float lse = 0.0f, logs = 0.0f;
  if (lane == 0) {
    logs = LN2 * log2f(st.s);
    lse = st.m == -INFINITY ? (st.s == 0.0f ? -INFINITY : NAN) : st.m + logs;
    a.lse[row] = lse;
    if (!(lse < INFINITY)) twa_set_status(a.status, TWA_ERR_NONFINITE, static_cast<int>(row));
    const bool none = lse == -INFINITY;
    if (ENT) a.entropy[row] = none ? 0.0f : logs - LN2 * (st.a / st.s);
    const long long t = twa_load_id(a.targets, a.itype, row);
    float lp = 0.0f;
    if (t != a.ignore_id) {
      if (t < 0 || t >= a.vocab) {
        twa_set_status(a.status, TWA_ERR_INVALID_ARG, static_cast<int>(row));
        lp = NAN;
      } else {
        lp = none ? -INFINITY : twa_to_float(x.base[x.skew + t]) - st.m - logs;
      }
    }
    a.logp[row] = lp;
  }
  if (TOP) {
    lse = __shfl_sync(0xffffffffu, lse, 0);
    logs = __shfl_sync(0xffffffffu, logs, 0);
    const float top = __shfl_sync(0xffffffffu, st.m, 0);
    if (lane < a.top) {
      a.top_ids[row * a.top + lane] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(found));
      a.top_logp[row * a.top + lane] = lse == -INFINITY ? -INFINITY : lp_unrank(static_cast<uint32_t>(found >> 32)) - top - logs;
    }
  }
}

constexpr int LPB_THREADS = 256;

// Rows x parts blocks; SAME: logits and dlogits rows lie alike on 16-byte boundaries, else element by element.
template <typename T, bool ENT, bool SAME>
__global__ void __launch_bounds__(LPB_THREADS) logprobs_backward_kernel(const LpArgs a, const int parts) {
  constexpr int E = twa_vec<T>;
  const long long row = blockIdx.x / parts;
  const int part = static_cast<int>(blockIdx.x - row * parts);
  const T* src = static_cast<const T*>(a.logits) + row * a.ld;
  T* dst = static_cast<T*>(a.dlogits) + row * a.ldd;
  const float lse = a.lse[row];
  const long long t = twa_load_id(a.targets, a.itype, row);
  const bool ignored = t == a.ignore_id, none = lse == -INFINITY;
  if (!ignored && (t < 0 || t >= a.vocab) && part == 0 && threadIdx.x == 0)
    twa_set_status(a.status, TWA_ERR_INVALID_ARG, static_cast<int>(row));
  const float dl = ignored || none ? 0.0f : a.d_logp[row];
  const float dh = ENT && !none ? a.d_entropy[row] : 0.0f, h = ENT ? a.entropy[row] : 0.0f;
  const float c = none ? 0.0f : lse;
  // dz = -p (dl + dh (log p + H)), and dl more at the target
  auto grad = [&](float z, int j) {
    const float d = (z - c) * LOG2E;
    float g = dl;
    if (ENT) g = fmaf(dh, fmaf(fmaxf(d, -150.0f), LN2, h), dl);
    const float o = -lp_exp2(d) * g;
    return j == t ? o + dl : o;
  };
  if (SAME) {
    const LpRow<T> x(src, a.vocab);
    const int units = x.units();
    T* out = dst - x.skew;
    for (int u = part * LPB_THREADS + threadIdx.x; u < units; u += parts * LPB_THREADS) {
      float v[E];
      if (x.whole(u)) {
        twa_pack<T, E> q;
        q.load(x.base + static_cast<long long>(u) * E);
        q.widen(v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = grad(v[e], u * E + e - x.skew);
        twa_pack<T, E>::store(out + static_cast<long long>(u) * E, v);
      } else {
        const unsigned valid = x.load_partial(u, v);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (valid >> e & 1) out[u * E + e] = twa_from_float<T>(grad(v[e], u * E + e - x.skew));
      }
    }
  } else {
    for (int j = part * LPB_THREADS + threadIdx.x; j < a.vocab; j += parts * LPB_THREADS)
      dst[j] = twa_from_float<T>(grad(twa_to_float(src[j]), j));
  }
}

template <typename T, bool ENT, bool TOP>
int lp_launch(twa_ctx* ctx, const LpArgs& a, int parts) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows * parts));
  cfg.blockDim = dim3(LP_THREADS);
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  TWA_CUDA_OK(ctx, cudaLaunchKernelEx(&cfg, logprobs_kernel<T, ENT, TOP>, a, parts));
  return TWA_OK;
}

template <typename T>
int lp_launch_any(twa_ctx* ctx, const LpArgs& a, int parts) {
  if (a.entropy) return a.top ? lp_launch<T, true, true>(ctx, a, parts) : lp_launch<T, true, false>(ctx, a, parts);
  return a.top ? lp_launch<T, false, true>(ctx, a, parts) : lp_launch<T, false, false>(ctx, a, parts);
}

template <typename T, bool ENT>
void lp_launch_backward(twa_ctx* ctx, const LpArgs& a, int parts, bool same) {
  const unsigned blocks = static_cast<unsigned>(a.rows * parts);
  if (same) logprobs_backward_kernel<T, ENT, true><<<blocks, LPB_THREADS, 0, ctx->stream>>>(a, parts);
  else logprobs_backward_kernel<T, ENT, false><<<blocks, LPB_THREADS, 0, ctx->stream>>>(a, parts);
}

int lp_check(const twa_ctx* ctx, twa_dtype dt, twa_itype it, int64_t rows, int vocab) {
  if (!ctx || !twa_dtype_ok(dt) || !twa_itype_ok(it) || rows < 0 || vocab < 1) return TWA_ERR_INVALID_ARG;
  if (rows > TWA_LOGPROBS_MAX_ROWS || vocab > TWA_LOGPROBS_MAX_VOCAB) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

}  // namespace

extern "C" {

int twa_token_logprobs(twa_ctx* ctx, const void* logits, int64_t ld, twa_dtype dtype, int64_t rows, int vocab,
                       const void* targets, twa_itype t_type, int64_t ignore_id, float* logp, float* lse, float* entropy,
                       int top, int32_t* top_ids, float* top_logp) {
  int rc = lp_check(ctx, dtype, t_type, rows, vocab);
  if (rc) return rc;
  if (top < 0 || top > vocab) return TWA_ERR_INVALID_ARG;
  if (top > TWA_LOGPROBS_MAX_TOP) return TWA_ERR_UNSUPPORTED;
  if (rows == 0) return TWA_OK;
  if (!logits || !targets || !logp || !lse || ld < vocab || (top && (!top_ids || !top_logp))) return TWA_ERR_INVALID_ARG;
  if (twa_misaligned_to(logits, twa_dtype_size(dtype)) || twa_misaligned_to(targets, twa_itype_size(t_type)) ||
      twa_misaligned_to(logp, 4) || twa_misaligned_to(lse, 4) || twa_misaligned_to(entropy, 4) || twa_misaligned_to(top_ids, 4) ||
      twa_misaligned_to(top_logp, 4))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LpArgs a = {};
  a.logits = logits;
  a.targets = targets;
  a.logp = logp;
  a.lse = lse;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_logp = top_logp;
  a.ld = ld;
  a.rows = rows;
  a.ignore_id = ignore_id;
  a.vocab = vocab;
  a.itype = t_type;
  a.top = top;
  a.status = ctx->d_status;
  int parts = 1;
  const long long units = twa_ceil_div(static_cast<long long>(vocab) * twa_dtype_size(dtype), 16);
  while (parts < LP_MAX_CLUSTER && rows * parts < ctx->sm_count && units > 2LL * LP_THREADS * parts) parts *= 2;
  return dtype == TWA_BF16 ? lp_launch_any<bf16>(ctx, a, parts) : lp_launch_any<float>(ctx, a, parts);
}

int twa_token_logprobs_backward(twa_ctx* ctx, const void* logits, int64_t ld, twa_dtype dtype, int64_t rows, int vocab,
                                const void* targets, twa_itype t_type, int64_t ignore_id, const float* lse,
                                const float* entropy, const float* d_logp, const float* d_entropy, void* dlogits, int64_t ldd) {
  int rc = lp_check(ctx, dtype, t_type, rows, vocab);
  if (rc) return rc;
  if (rows == 0) return TWA_OK;
  if (!logits || !targets || !lse || !d_logp || !dlogits || ld < vocab || ldd < vocab || (d_entropy && !entropy))
    return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(logits, size) || twa_misaligned_to(dlogits, size) || twa_misaligned_to(targets, twa_itype_size(t_type)) ||
      twa_misaligned_to(lse, 4) || twa_misaligned_to(entropy, 4) || twa_misaligned_to(d_logp, 4) || twa_misaligned_to(d_entropy, 4))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LpArgs a = {};
  a.logits = logits;
  a.targets = targets;
  a.lse = const_cast<float*>(lse);
  a.entropy = const_cast<float*>(entropy);
  a.d_logp = d_logp;
  a.d_entropy = d_entropy;
  a.dlogits = dlogits;
  a.ld = ld;
  a.ldd = ldd;
  a.rows = rows;
  a.ignore_id = ignore_id;
  a.vocab = vocab;
  a.itype = t_type;
  a.status = ctx->d_status;
  const bool same = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15) == 0 &&
                    (rows == 1 || ((ld - ldd) * static_cast<int64_t>(size)) % 16 == 0);
  const long long units = twa_ceil_div(static_cast<long long>(vocab) * size, 16);
  long long parts = twa_ceil_div(units, 8LL * LPB_THREADS);
  while (parts < twa_ceil_div(units, LPB_THREADS) && rows * parts < 4LL * ctx->sm_count) ++parts;
  if (rows * parts > 0x7fffffffLL) return TWA_ERR_UNSUPPORTED;
  if (dtype == TWA_BF16) {
    if (d_entropy) lp_launch_backward<bf16, true>(ctx, a, static_cast<int>(parts), same);
    else lp_launch_backward<bf16, false>(ctx, a, static_cast<int>(parts), same);
  } else {
    if (d_entropy) lp_launch_backward<float, true>(ctx, a, static_cast<int>(parts), same);
    else lp_launch_backward<float, false>(ctx, a, static_cast<int>(parts), same);
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
