// Tokens sorted by expert, and the experts' results brought back with weights.
//
//   dispatch           the assignments (t, j), j < top, sorted by their expert, equal ones in the order of t and j;
//                      out[place[t, j]] = x[t]
//   combine            out[t] = sum_j w[t, j] y[place[t, j]], added in the order of j
//   combine backward   dy[place[t, j]] = w[t, j] dout[t],   dw[t, j] = sum dout[t] y[place[t, j]]
//
// The sort is a counting sort by one cluster of blocks in its shared memory, one launch whatever the number: every warp has a
// run of assignments and counts them by expert, 32 at a time (lanes of the same expert find each other by a match, the first of
// them adds their number), a prefix over warps, blocks and experts gives every warp its first place for every expert, and a
// second walk gives places out.  No count depends on which block came first.  What moves rows is bound by memory and
// goes token by token, so that a token's row is read, or written, once for all its experts.
#include "twa_ops.cuh"

namespace {

// ---- the sort -----------------------------------------------------------------------------------
constexpr int SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_LOADS = 4;                     // ids of a lane under way together

struct SortArgs {
  const void* ids;
  int itype;
  long long tokens;
  int count, top, experts;                        // count: assignments
  int warps;                                      // of a block that take part (shared memory holds a count of each expert for each)
  int run;                                        // assignments of a warp
  int* place;
  int* order;
  int* starts;
  int* status;
};

// Expert of an assignment, -1 for none.
__device__ __forceinline__ int expert_of(const SortArgs& a, long long i, bool report) {
  const long long id = twa_load_id(a.ids, a.itype, i);
  if (id >= 0 && id < a.experts) return static_cast<int>(id);
  if (report && id != -1) twa_set_status(a.status, TWA_ERR_INVALID_ARG, static_cast<int>(i / a.top));
  return -1;
}

__global__ void __launch_bounds__(SORT_THREADS) expert_sort_kernel(SortArgs a, int blocks) {
  twa_begin(a.ids);
  extern __shared__ int shared[];
  int* total = shared;                            // of this block, by expert
  int* base = total + a.experts;                  // place of this block's first assignment of an expert
  int* count = base + a.experts;                  // [warps][experts]
  const int rank = blocks > 1 ? static_cast<int>(twa_cluster_rank()) : 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < a.warps * a.experts; i += SORT_THREADS) count[i] = 0;
  __syncthreads();
  const long long from = static_cast<long long>(rank * a.warps + warp) * a.run;
  const int first = warp < a.warps && from < a.count ? static_cast<int>(from) : a.count;
  const int last = a.count - first < a.run ? a.count : first + a.run;
  int* mine = count + (warp < a.warps ? warp * a.experts : 0);
  for (int i = first; i < last; i += 32 * SORT_LOADS) {
    int e[SORT_LOADS];
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k) e[k] = i + k * 32 + lane < last ? expert_of(a, i + k * 32 + lane, true) : -1;
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k) {
      const unsigned same = __match_any_sync(0xffffffffu, e[k]);
      if (e[k] >= 0 && (same & ((1u << lane) - 1)) == 0) mine[e[k]] += __popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += SORT_THREADS) {
    int sum = 0;
    for (int w = 0; w < a.warps; ++w) {
      const int c = count[w * a.experts + e];
      count[w * a.experts + e] = sum;
      sum += c;
    }
    total[e] = sum;
  }
  if (blocks > 1) twa_cluster_sync();
  else __syncthreads();
  // assignments of every expert in all blocks, and of them those in blocks before this one
  int* all = count + a.warps * a.experts;
  for (int e = threadIdx.x; e < a.experts; e += SORT_THREADS) {
    int before = 0, sum = 0;
    for (int r = 0; r < blocks; ++r) {
      const int c = r == rank ? total[e] : twa_remote(total + e, r);
      before += r < rank ? c : 0;
      sum += c;
    }
    base[e] = before;
    all[e] = sum;
  }
  if (blocks > 1) twa_cluster_sync();             // no block ends while another reads its totals
  else __syncthreads();
  if (warp == 0) {
    int sum = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 32) {
      const int e = e0 + lane, c = e < a.experts ? all[e] : 0;
      int upto = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      if (e < a.experts) {
        base[e] += sum + upto - c;
        if (rank == 0) a.starts[e] = sum + upto - c;
      }
      sum += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (rank == 0 && lane == 0) a.starts[a.experts] = sum;
  }
  __syncthreads();
  for (int i = first; i < last; i += 32 * SORT_LOADS) {
    int e[SORT_LOADS];
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k) e[k] = i + k * 32 + lane < last ? expert_of(a, i + k * 32 + lane, false) : -1;
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k) {
      const int n = i + k * 32 + lane;
      const unsigned same = __match_any_sync(0xffffffffu, e[k]), before = same & ((1u << lane) - 1);
      const int at = e[k] >= 0 ? base[e[k]] + mine[e[k]] + __popc(before) : -1;
      __syncwarp();
      if (e[k] >= 0 && before == 0) mine[e[k]] += __popc(same);
      __syncwarp();
      if (n < last) {
        a.place[n] = at;
        if (a.order && at >= 0) a.order[at] = n;
      }
    }
  }
}

// ---- rows to their experts ------------------------------------------------------------------------
constexpr int MOVE_WARPS = 8;

// A warp takes UNITS x 32 units of a token's row, as bytes.
template <typename W, int UNITS>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_gather_kernel(const char* x, long long ldx, long long tokens, int units, int parts,
                                                                         const int* place, int top, char* out, long long ldo) {
  twa_begin(x, place);
  const long long task = static_cast<long long>(blockIdx.x) * MOVE_WARPS + (threadIdx.x >> 5);
  const long long t = task / parts;
  if (t >= tokens) return;
  const int lane = threadIdx.x & 31, u0 = static_cast<int>(task - t * parts) * (UNITS * 32) + lane;
  const int mine = lane < top ? __ldg(place + t * top + lane) : -1;
  const W* from = reinterpret_cast<const W*>(x + t * ldx);
  W v[UNITS];
#pragma unroll
  for (int k = 0; k < UNITS; ++k)
    if (u0 + k * 32 < units) v[k] = __ldg(from + u0 + k * 32);
  for (int j = 0; j < top; ++j) {
    const int p = __shfl_sync(0xffffffffu, mine, j);
    if (p < 0) continue;
    W* to = reinterpret_cast<W*>(out + p * ldo);
#pragma unroll
    for (int k = 0; k < UNITS; ++k)
      if (u0 + k * 32 < units) to[u0 + k * 32] = v[k];
  }
}

// ---- and back ---------------------------------------------------------------------------------------
struct CombineArgs {
  const void* y;
  const void* dout;
  const int* place;
  const float* weights;
  void* out;                                      // or dy
  float* dw;
  long long ldy, ldd, ldo, rows, tokens;
  int top, dim, parts;
  int* status;
};

// Place of assignment i: -1 for none and, reported, for one outside the rows.
__device__ __forceinline__ int place_of(const CombineArgs& a, long long t, int j, bool report) {
  const int p = __ldg(a.place + t * a.top + j);
  if (p >= a.rows) {
    if (report) twa_set_status(a.status, TWA_ERR_INVALID_ARG, static_cast<int>(t));
    return -1;
  }
  return p;
}

constexpr int COMBINE_LOADS = 4;                  // rows of a token under way together
template <typename T, int E>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_combine_kernel(CombineArgs a) {
  twa_begin(a.y, a.place, a.weights);
  const long long task = static_cast<long long>(blockIdx.x) * MOVE_WARPS + (threadIdx.x >> 5);
  const long long t = task / a.parts;
  if (t >= a.tokens) return;
  const int lane = threadIdx.x & 31, part = static_cast<int>(task - t * a.parts), c = (part * 32 + lane) * E;
  const int place = lane < a.top ? place_of(a, t, lane, part == 0) : -1;
  const float weight = lane < a.top ? (a.weights ? __ldg(a.weights + t * a.top + lane) : 1.0f) : 0.0f;
  const T* y = static_cast<const T*>(a.y) + c;
  float sum[E] = {};
  for (int j0 = 0; j0 < a.top; j0 += COMBINE_LOADS) {
    twa_pack<T, E> raw[COMBINE_LOADS];
    int p[COMBINE_LOADS];
#pragma unroll
    for (int k = 0; k < COMBINE_LOADS; ++k) {
      p[k] = __shfl_sync(0xffffffffu, place, (j0 + k) & 31);
      if (j0 + k >= a.top || c >= a.dim) p[k] = -1;
      if (p[k] >= 0) raw[k].load(y + p[k] * a.ldy);
    }
#pragma unroll
    for (int k = 0; k < COMBINE_LOADS; ++k) {
      const float w = __shfl_sync(0xffffffffu, weight, (j0 + k) & 31);
      if (p[k] < 0) continue;
      float v[E];
      raw[k].widen(v);
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] = fmaf(w, v[e], sum[e]);
    }
  }
  if (c < a.dim) twa_pack<T, E>::store(static_cast<T*>(a.out) + t * a.ldo + c, sum);
}

// A token's row for a group of LANES threads (a warp, or the block): the dot products need the whole row.  BATCH experts at a time.
constexpr int BACK_BATCH = 4;
template <typename T, int E, int LANES>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_combine_backward_kernel(CombineArgs a) {
  twa_begin(a.y, a.dout, a.place, a.weights);
  __shared__ float part[LANES > 32 ? MOVE_WARPS : 1][32];
  const long long t = LANES > 32 ? blockIdx.x : static_cast<long long>(blockIdx.x) * MOVE_WARPS + (threadIdx.x >> 5);
  if (t >= a.tokens) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = LANES > 32 ? threadIdx.x : lane;
  const int place = lane < a.top ? place_of(a, t, lane, warp == 0 || LANES == 32) : -1;
  const float weight = lane < a.top ? __ldg(a.weights + t * a.top + lane) : 0.0f;
  const T* dout = static_cast<const T*>(a.dout) + t * a.ldd;
  for (int j0 = 0; j0 < a.top; j0 += BACK_BATCH) {
    int p[BACK_BATCH];
    float w[BACK_BATCH], dot[BACK_BATCH];
#pragma unroll
    for (int k = 0; k < BACK_BATCH; ++k) {
      p[k] = __shfl_sync(0xffffffffu, place, (j0 + k) & 31);
      w[k] = __shfl_sync(0xffffffffu, weight, (j0 + k) & 31);
      if (j0 + k >= a.top) p[k] = -1;
      dot[k] = 0.0f;
    }
    for (int c = at * E; c < a.dim; c += LANES * E) {
      twa_pack<T, E> rd, ry[BACK_BATCH];
      rd.load(dout + c);
#pragma unroll
      for (int k = 0; k < BACK_BATCH; ++k)
        if (p[k] >= 0) ry[k].load(static_cast<const T*>(a.y) + p[k] * a.ldy + c);
      float d[E];
      rd.widen(d);
#pragma unroll
      for (int k = 0; k < BACK_BATCH; ++k) {
        if (p[k] < 0) continue;
        float v[E];
        ry[k].widen(v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          dot[k] = fmaf(d[e], v[e], dot[k]);
          v[e] = w[k] * d[e];
        }
        twa_pack<T, E>::store(static_cast<T*>(a.out) + p[k] * a.ldo + c, v);
      }
    }
#pragma unroll
    for (int k = 0; k < BACK_BATCH; ++k) {
      const float sum = twa_warp_sum(dot[k]);
      if (LANES > 32) {
        if (lane == 0 && j0 + k < a.top) part[warp][j0 + k] = sum;
      } else if (a.dw && lane == 0 && j0 + k < a.top) {
        a.dw[t * a.top + j0 + k] = sum;
      }
    }
  }
  if (LANES > 32 && a.dw) {
    __syncthreads();
    if (threadIdx.x < a.top) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < MOVE_WARPS; ++w) sum += part[w][threadIdx.x];
      a.dw[t * a.top + threadIdx.x] = sum;
    }
  }
}

bool on_unit(const void* p, long long ld_bytes, size_t unit) { return !twa_misaligned_to(p, unit) && ld_bytes % unit == 0; }

template <typename W, int UNITS>
void launch_gather(twa_ctx* ctx, const void* x, long long ldx, long long tokens, long long bytes, const int* place, int top, void* out,
                   long long ldo) {
  const int units = static_cast<int>(bytes / sizeof(W)), parts = static_cast<int>(twa_ceil_div(units, UNITS * 32));
  twa_launch(ctx->stream, expert_gather_kernel<W, UNITS>, static_cast<unsigned>(twa_ceil_div(tokens * parts, MOVE_WARPS)), MOVE_WARPS * 32, 0,
             static_cast<const char*>(x), ldx, tokens, units, parts, place, top, static_cast<char*>(out), ldo);
}

int expert_sizes(twa_ctx* ctx, int64_t tokens, int top) {
  if (!ctx || tokens < 0 || top < 1) return TWA_ERR_INVALID_ARG;
  if (top > TWA_EXPERTS_MAX_TOP || tokens > TWA_EXPERTS_MAX_ASSIGNMENTS / top) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

template <typename T>
void launch_combine(twa_ctx* ctx, CombineArgs a, bool packs) {
  constexpr int V = twa_vec<T>;
  a.parts = static_cast<int>(twa_ceil_div(a.dim, 32 * (packs ? V : 1)));
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.tokens * a.parts, MOVE_WARPS));
  if (packs) twa_launch(ctx->stream, expert_combine_kernel<T, V>, blocks, MOVE_WARPS * 32, 0, a);
  else twa_launch(ctx->stream, expert_combine_kernel<T, 1>, blocks, MOVE_WARPS * 32, 0, a);
}

template <typename T, int E>
void launch_combine_backward(twa_ctx* ctx, const CombineArgs& a) {
  if (a.tokens >= 16LL * ctx->sm_count)
    twa_launch(ctx->stream, expert_combine_backward_kernel<T, E, 32>, static_cast<unsigned>(twa_ceil_div(a.tokens, MOVE_WARPS)), MOVE_WARPS * 32,
               0, a);
  else
    twa_launch(ctx->stream, expert_combine_backward_kernel<T, E, MOVE_WARPS * 32>, static_cast<unsigned>(a.tokens), MOVE_WARPS * 32, 0, a);
}

}  // namespace

extern "C" {

int twa_expert_dispatch(twa_ctx* ctx, const void* x, int64_t ldx, twa_dtype dtype, int64_t tokens, int dim, const void* ids, twa_itype id_type,
                        int top, int experts, int32_t* place, int32_t* starts, int32_t* order, void* out, int64_t ldo) {
  int rc = expert_sizes(ctx, tokens, top);
  if (rc) return rc;
  if (!twa_dtype_ok(dtype) || !twa_itype_ok(id_type) || experts < 1 || dim < 1) return TWA_ERR_INVALID_ARG;
  if (experts > TWA_EXPERTS_MAX || dim > TWA_EXPERTS_MAX_DIM) return TWA_ERR_UNSUPPORTED;
  if (!starts || (tokens && (!ids || !place)) || !x != !out) return TWA_ERR_INVALID_ARG;
  if (x && tokens && (ldx < dim || ldo < dim)) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(starts, 4) || (tokens && (twa_misaligned_to(ids, twa_itype_size(id_type)) || twa_misaligned_to(place, 4) ||
                                                  twa_misaligned_to(order, 4) || twa_misaligned_to(x, size) || twa_misaligned_to(out, size))))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  SortArgs s = {ids, id_type, tokens, static_cast<int>(tokens * top), top, experts, SORT_WARPS, 0, place, order, starts, ctx->d_status};
  while (s.warps > 1 && sizeof(int) * (s.warps + 3) * experts > 48 * 1024) s.warps /= 2;
  int blocks = 1;
  while (blocks < 8 && s.count > blocks * s.warps * 32 * SORT_LOADS) blocks *= 2;
  s.run = static_cast<int>(twa_ceil_div(twa_ceil_div(s.count, blocks * s.warps), 32) * 32);
  TWA_CUDA_OK(ctx, twa_launch_clusters(ctx->stream, expert_sort_kernel, blocks, blocks, SORT_THREADS, sizeof(int) * (s.warps + 3) * experts, s,
                                       blocks));
  if (x && tokens) {
    const long long bytes = static_cast<long long>(dim) * size, lx = ldx * size, lo = ldo * size;
    const bool wide = bytes % 16 == 0 && on_unit(x, lx, 16) && on_unit(out, lo, 16);
    if (wide) launch_gather<uint4, 4>(ctx, x, lx, tokens, bytes, place, top, out, lo);
    else if (bytes % 4 == 0 && on_unit(x, lx, 4) && on_unit(out, lo, 4)) launch_gather<uint32_t, 8>(ctx, x, lx, tokens, bytes, place, top, out, lo);
    else launch_gather<unsigned short, 8>(ctx, x, lx, tokens, bytes, place, top, out, lo);
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

int twa_expert_combine(twa_ctx* ctx, const void* y, int64_t ldy, twa_dtype dtype, int64_t rows, const int32_t* place, const float* weights,
                       int64_t tokens, int top, int dim, void* out, int64_t ldo) {
  int rc = expert_sizes(ctx, tokens, top);
  if (rc) return rc;
  if (!twa_dtype_ok(dtype) || rows < 0 || dim < 1) return TWA_ERR_INVALID_ARG;
  if (dim > TWA_EXPERTS_MAX_DIM) return TWA_ERR_UNSUPPORTED;
  if (tokens == 0) return TWA_OK;
  if (!place || !out || ldo < dim || (rows && (!y || ldy < dim))) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(place, 4) || twa_misaligned_to(weights, 4) || twa_misaligned_to(out, size) || (rows && twa_misaligned_to(y, size)))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  const bool packs = dim * size % 16 == 0 && on_unit(y, ldy * size, 16) && on_unit(out, ldo * size, 16);
  CombineArgs a = {y, nullptr, place, weights, out, nullptr, ldy, 0, ldo, rows, tokens, top, dim, 0, ctx->d_status};
  if (dtype == TWA_BF16) launch_combine<bf16>(ctx, a, packs);
  else launch_combine<float>(ctx, a, packs);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

int twa_expert_combine_backward(twa_ctx* ctx, const void* dout, int64_t lddout, const void* y, int64_t ldy, twa_dtype dtype, int64_t rows,
                                const int32_t* place, const float* weights, int64_t tokens, int top, int dim, void* dy, int64_t lddy,
                                float* dw) {
  int rc = expert_sizes(ctx, tokens, top);
  if (rc) return rc;
  if (!twa_dtype_ok(dtype) || rows < 0 || dim < 1) return TWA_ERR_INVALID_ARG;
  if (dim > TWA_EXPERTS_MAX_DIM) return TWA_ERR_UNSUPPORTED;
  if (tokens == 0) return TWA_OK;
  if (!dout || lddout < dim || !place || !weights || (rows && (!y || ldy < dim || !dy || lddy < dim))) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(dout, size) || twa_misaligned_to(place, 4) || twa_misaligned_to(weights, 4) || twa_misaligned_to(dw, 4) ||
      (rows && (twa_misaligned_to(y, size) || twa_misaligned_to(dy, size))))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  const bool packs = dim * size % 16 == 0 && on_unit(dout, lddout * size, 16) && on_unit(y, ldy * size, 16) && on_unit(dy, lddy * size, 16);
  const CombineArgs a = {y, dout, place, weights, dy, dw, ldy, lddout, lddy, rows, tokens, top, dim, 0, ctx->d_status};
  if (dtype == TWA_BF16) {
    if (packs) launch_combine_backward<bf16, 8>(ctx, a);
    else launch_combine_backward<bf16, 1>(ctx, a);
  } else {
    if (packs) launch_combine_backward<float, 4>(ctx, a);
    else launch_combine_backward<float, 1>(ctx, a);
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
