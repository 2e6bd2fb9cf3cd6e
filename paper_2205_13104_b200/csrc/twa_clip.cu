// The norm of all gradients together, and clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2),   factor = min(1, max_norm / (norm + eps)),   out = factor g
//
// The gradients lie in many tensors of different sizes, addresses and types; the result is the flat vector that a
// subspace step takes, or the tensors themselves.  One kernel adds the squares, one scales; both are bound by memory, and
// the gradients are read twice because the factor depends on all of them.  The second kernel walks backwards, so that
// what the first read last is found in L2.
//
// The tensors' addresses travel as kernel arguments (CLIP_TENSORS of them a launch), so a call uploads nothing.  They are
// cut into chunks of at most CLIP_CHUNK elements; a block takes a run of chunks of equal length in either kernel.
// 86.6 M float32 in 152 tensors: 195 us, 1.04 GB at 5.3 TB/s (60 us the norm); 1.32 G bfloat16 in 388: 1280 to 1306 us, 7.9 GB at
// 6.1 TB/s; 400 M bfloat16 in 388 tensors of odd sizes, of which most lie on other boundaries than their place in the flat vector and
// are scaled element by element: 527 us, 2.4 GB at 4.6 TB/s.
// With chunks dealt out to the blocks in turn 700 small tensors take 72 us instead of 38; streaming stores change nothing.
//
// Squares are added in float32 over the elements of one load and in float64 beyond, in a fixed order.  Where that left float32, or a
// load's squares are so small that they have lost digits, the thread takes its part of the chunk once more in float64 (a
// branch at each load instead: 86.6 M float32 199 -> 224 us, 1.32 G bfloat16 1293 -> 2030).
#include <math.h>

#include "twa_ops.cuh"

namespace {

constexpr int CLIP_TENSORS = 512;       // tensors of one launch
constexpr int CLIP_FEW = 32;            // a smaller table, which costs less to hand over (10 tensors: 8.5 us a call, else 11.4)
constexpr int CLIP_CHUNK = 8192;        // elements
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_SM_BLOCKS = 5;       // blocks an SM (86.6 M float32: 196 us, 4 blocks 201)
constexpr int CLIP_MAX_BLOCKS = 148 * 8;
constexpr int CLIP_HEAD = 256;          // bytes of the workspace before the partial sums: the factor

template <int N>
struct ClipTable {
  const void* data[N];
  long long flat[N + 1];                // where the tensor begins in the flat vector, and where the last one ends
  int chunk[N + 1];                     // first chunk of each tensor, and the number of chunks
  unsigned char dtype[N];
  int count;
};

// Tensor that chunk q belongs to.
template <int N>
__device__ __forceinline__ int clip_find(const ClipTable<N>& t, int q) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.chunk[mid] <= q) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Below this a load's squares may have lost digits: each errs by 2^-150 at most, which is 2^-27 of such a sum of eight.
constexpr float CLIP_SMALL = 0x1p-120f;

// Bits that are set in any element, signs aside.
__device__ __forceinline__ uint32_t clip_bits(const twa_pack<float, 4>& q) {
  return (__float_as_uint(q.r.x) | __float_as_uint(q.r.y) | __float_as_uint(q.r.z) | __float_as_uint(q.r.w)) & 0x7fffffffu;
}
__device__ __forceinline__ uint32_t clip_bits(const twa_pack<bf16, 8>& q) { return (q.r.x | q.r.y | q.r.z | q.r.w) & 0x7fff7fffu; }

// A chunk as elements before the first 16-byte boundary (`head` of them), units of 16 bytes, and the rest from `tail` on.
template <typename T>
struct ClipParts {
  static constexpr int E = twa_vec<T>;
  int head, units, tail;
  __device__ __forceinline__ ClipParts(const T* p, int n) {
    const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    head = min(n, skew ? E - skew : 0);
    units = (n - head) / E;
    tail = head + units * E;
  }
};

// What clip_square_sum gives, every square in float64.
template <typename T>
__device__ __noinline__ double clip_square_sum_wide(const T* p, int n) {
  const ClipParts<T> parts(p, n);
  const int t = threadIdx.x;
  double sum = 0.0;
  auto square = [&](int i) {
    const double v = twa_to_float(p[i]);
    sum += v * v;
  };
  if (t < parts.head) square(t);
  if (parts.tail + t < n) square(parts.tail + t);
  for (int u = t; u < parts.units; u += CLIP_THREADS)
    for (int e = 0; e < parts.E; ++e) square(parts.head + u * parts.E + e);
  return sum;
}

// The squares of a thread's elements of a chunk.
template <typename T>
__device__ __forceinline__ double clip_square_sum(const T* p, int n) {
  constexpr int E = twa_vec<T>;
  double sum = 0.0;
  uint32_t small = 0;                   // bits of elements whose squares have lost digits
  const ClipParts<T> parts(p, n);
  const int head = parts.head, units = parts.units, tail = parts.tail;
  if (static_cast<int>(threadIdx.x) < head) {
    const double v = twa_to_float(p[threadIdx.x]);
    sum += v * v;
  }
  if (tail + static_cast<int>(threadIdx.x) < n) {
    const double v = twa_to_float(p[tail + threadIdx.x]);
    sum += v * v;
  }
  constexpr int AHEAD = 4;
  const T* from = p + head + threadIdx.x * E;
  int left = units - static_cast<int>(threadIdx.x);
  auto squares = [&](const twa_pack<T, E>& q) {
    float v[E], s = 0.0f;
    q.widen(v);
#pragma unroll
    for (int e = 0; e < E; ++e) s += v[e] * v[e];
    sum += static_cast<double>(s);
    if (s < CLIP_SMALL) small |= clip_bits(q);
  };
  for (; left > (AHEAD - 1) * CLIP_THREADS; left -= AHEAD * CLIP_THREADS) {
    twa_pack<T, E> q[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) q[k].load(from + k * CLIP_THREADS * E);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) squares(q[k]);
    from += AHEAD * CLIP_THREADS * E;
  }
#pragma unroll 1
  for (; left > 0; left -= CLIP_THREADS) {
    twa_pack<T, E> q;
    q.load(from);
    squares(q);
    from += CLIP_THREADS * E;
  }
  return small || !isfinite(sum) ? clip_square_sum_wide(p, n) : sum;
}

__device__ __forceinline__ double clip_block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
  for (int k = 0; k < CLIP_THREADS / 32; ++k) v += red[k];
  __syncthreads();
  return v;
}

// Partial sums of this launch's tensors to part[base + block]; the last block of the last launch adds all `total` of them.
template <int N>
__global__ void __launch_bounds__(CLIP_THREADS, CLIP_SM_BLOCKS) clip_norm_kernel(const __grid_constant__ ClipTable<N> t, double* part, int base, int total, unsigned* ticket, float max_norm, float eps,
                                                                 float* norm_out, float* factor, int* status) {
  twa_begin(part, ticket, norm_out, factor);
  __shared__ double red[CLIP_THREADS / 32];
  __shared__ unsigned last;
  const int chunks = t.chunk[t.count];
  const int from = static_cast<int>(static_cast<long long>(chunks) * blockIdx.x / gridDim.x);
  const int to = static_cast<int>(static_cast<long long>(chunks) * (blockIdx.x + 1) / gridDim.x);
  double sum = 0.0;
  int i = from < to ? clip_find(t, from) : 0;
  for (int q = from; q < to; ++q) {
    while (t.chunk[i + 1] <= q) ++i;
    const long long off = static_cast<long long>(q - t.chunk[i]) * CLIP_CHUNK;
    const int n = static_cast<int>(min(static_cast<long long>(CLIP_CHUNK), t.flat[i + 1] - t.flat[i] - off));
    const void* data = t.data[i];
    twa_renew(data);
    sum += t.dtype[i] == TWA_BF16 ? clip_square_sum(static_cast<const bf16*>(data) + off, n)
                                  : clip_square_sum(static_cast<const float*>(data) + off, n);
  }
  sum = clip_block_sum(sum, red);
  if (threadIdx.x == 0) part[base + blockIdx.x] = sum;
  if (total == 0) return;
  __threadfence();
  if (threadIdx.x == 0) last = atomicAdd(ticket, 1u);
  __syncthreads();
  if (last != gridDim.x - 1) return;
  __threadfence();
  double all = 0.0;
  for (int k = threadIdx.x; k < total; k += CLIP_THREADS) all += __ldcg(part + k);
  all = clip_block_sum(all, red);
  if (threadIdx.x == 0) {
    *ticket = 0;
    const double norm = sqrt(all);
    const float rounded = static_cast<float>(norm);
    *norm_out = rounded;
    const double f = static_cast<double>(max_norm) / (norm + static_cast<double>(eps));
    if (factor) *factor = static_cast<float>(f >= 1.0 ? 1.0 : f);      // a norm that is no number gives none
    if (!isfinite(rounded)) twa_set_status(status, TWA_ERR_NONFINITE, -1);
  }
}

// 8 elements of a thread and AHEAD such loads under way at once where both lie on 16 bytes, else element by element, SINGLY loads
// at once.
template <typename T, typename TO>
__device__ __forceinline__ void clip_scale(const T* p, TO* o, int n, float f) {
  constexpr int E = 8, PACK = twa_vec<T>, PACKS = E / PACK, AHEAD = 4 / PACKS, SINGLY = 8;
  typedef twa_pack<T, PACK> Pack;
  auto eight = [&](const Pack (&q)[PACKS], TO* to) {
    float v[E];
#pragma unroll
    for (int k = 0; k < PACKS; ++k) q[k].widen(v + k * PACK);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= f;
#pragma unroll
    for (int k = 0; k < E; k += twa_vec<TO>) twa_pack<TO, twa_vec<TO>>::store(to + k, v + k);
  };
  int j = threadIdx.x;
  if (((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(o)) & 15) == 0) {
    const int units = n / E;
    const T* from = p + threadIdx.x * E;
    TO* to = o + threadIdx.x * E;
    int left = units - static_cast<int>(threadIdx.x);
    for (; left > (AHEAD - 1) * CLIP_THREADS; left -= AHEAD * CLIP_THREADS) {
      Pack q[AHEAD][PACKS];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
#pragma unroll
        for (int k = 0; k < PACKS; ++k) q[i][k].load(from + i * CLIP_THREADS * E + k * PACK);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) eight(q[i], to + i * CLIP_THREADS * E);
      from += AHEAD * CLIP_THREADS * E;
      to += AHEAD * CLIP_THREADS * E;
    }
#pragma unroll 1
    for (; left > 0; left -= CLIP_THREADS) {
      Pack q[PACKS];
#pragma unroll
      for (int k = 0; k < PACKS; ++k) q[k].load(from + k * PACK);
      eight(q, to);
      from += CLIP_THREADS * E;
      to += CLIP_THREADS * E;
    }
    j += units * E;
  }
  const T* from = p + j;
  TO* to = o + j;
  int left = n - j;
  for (; left > (SINGLY - 1) * CLIP_THREADS; left -= SINGLY * CLIP_THREADS) {
    twa_pack<T, 1> q[SINGLY];
#pragma unroll
    for (int i = 0; i < SINGLY; ++i) q[i].load(from + i * CLIP_THREADS);
#pragma unroll
    for (int i = 0; i < SINGLY; ++i) {
      float v[1];
      q[i].widen(v);
      to[i * CLIP_THREADS] = twa_from_float<TO>(v[0] * f);
    }
    from += SINGLY * CLIP_THREADS;
    to += SINGLY * CLIP_THREADS;
  }
#pragma unroll 1
  for (; left > 0; left -= CLIP_THREADS) {
    *to = twa_from_float<TO>(twa_to_float(*from) * f);
    from += CLIP_THREADS;
    to += CLIP_THREADS;
  }
}

// out == null: in place.
template <int N>
__global__ void __launch_bounds__(CLIP_THREADS, CLIP_SM_BLOCKS) clip_scale_kernel(const __grid_constant__ ClipTable<N> t, const float* __restrict__ factor,
                                                                  void* out, int out_dtype) {
  twa_begin(factor, out);
  const float f = __ldg(factor);
  if (!out && f == 1.0f) return;
  const int chunks = t.chunk[t.count], block = gridDim.x - 1 - blockIdx.x;
  const int from = static_cast<int>(static_cast<long long>(chunks) * block / gridDim.x);
  const int to = static_cast<int>(static_cast<long long>(chunks) * (block + 1) / gridDim.x);
  int i = from < to ? clip_find(t, to - 1) : 0;
  for (int q = to - 1; q >= from; --q) {
    while (t.chunk[i] > q) --i;
    const long long off = static_cast<long long>(q - t.chunk[i]) * CLIP_CHUNK;
    const int n = static_cast<int>(min(static_cast<long long>(CLIP_CHUNK), t.flat[i + 1] - t.flat[i] - off));
    const long long at = t.flat[i] + off;
    void* data = const_cast<void*>(t.data[i]);
    twa_renew(data);
    if (t.dtype[i] == TWA_BF16) {
      bf16* p = static_cast<bf16*>(data) + off;
      if (!out) clip_scale(p, p, n, f);
      else if (out_dtype == TWA_BF16) clip_scale(p, static_cast<bf16*>(out) + at, n, f);
      else clip_scale(p, static_cast<float*>(out) + at, n, f);
    } else {
      float* p = static_cast<float*>(data) + off;
      if (!out) clip_scale(p, p, n, f);
      else if (out_dtype == TWA_BF16) clip_scale(p, static_cast<bf16*>(out) + at, n, f);
      else clip_scale(p, static_cast<float*>(out) + at, n, f);
    }
  }
}

int clip_check(const twa_ctx* ctx, const twa_tensors* t) {
  if (!ctx || !t || t->count < 0 || (t->count && (!t->data || !t->sizes || !t->dtypes))) return TWA_ERR_INVALID_ARG;
  if (t->count > TWA_MAX_TENSORS) return TWA_ERR_UNSUPPORTED;
  long long total = 0;
  for (int i = 0; i < t->count; ++i) {
    if (t->sizes[i] < 0 || !twa_dtype_ok(t->dtypes[i]) || (t->sizes[i] && !t->data[i])) return TWA_ERR_INVALID_ARG;
    if (t->sizes[i] > TWA_MAX_ROWS || (total += t->sizes[i]) > TWA_MAX_ROWS) return TWA_ERR_UNSUPPORTED;
    if (t->sizes[i] && twa_misaligned_to(t->data[i], twa_dtype_size(t->dtypes[i]))) return TWA_ERR_MISALIGNED;
  }
  return TWA_OK;
}

// Fills the table of one launch from tensor `first` on; returns the first tensor that is not in it.
template <int N>
int clip_fill(const twa_tensors* s, int first, long long* flat, ClipTable<N>* t) {
  int i = first;
  t->count = 0;
  t->chunk[0] = 0;
  for (; i < s->count && t->count < N; ++i) {
    const long long n = s->sizes[i];
    if (!n) continue;
    const int k = t->count++;
    t->data[k] = s->data[i];
    t->flat[k] = *flat;
    t->dtype[k] = static_cast<unsigned char>(s->dtypes[i]);
    t->chunk[k + 1] = t->chunk[k] + static_cast<int>(twa_ceil_div(n, CLIP_CHUNK));
    *flat += n;
    t->flat[k + 1] = *flat;
  }
  return i;
}

int clip_blocks(const twa_ctx* ctx, int chunks) {
  int most = CLIP_SM_BLOCKS * ctx->sm_count;
  if (most > CLIP_MAX_BLOCKS) most = CLIP_MAX_BLOCKS;
  return chunks < 1 ? 1 : (chunks < most ? chunks : most);
}

template <int N>
int clip_run(twa_ctx* ctx, const twa_tensors* s, float max_norm, float eps, bool scale, void* out, int out_dtype, float* norm,
             void* ws) {
  float* factor = static_cast<float*>(ws);
  double* part = reinterpret_cast<double*>(static_cast<char*>(ws) + CLIP_HEAD);
  ClipTable<N> t;
  int base = 0, next = 0, launches = 0;
  long long flat = 0;
  do {
    next = clip_fill(s, next, &flat, &t);
    const int blocks = clip_blocks(ctx, t.chunk[t.count]);
    TWA_CUDA_OK(ctx, twa_launch(ctx->stream, clip_norm_kernel<N>, blocks, CLIP_THREADS, 0, t, part, base,
                                next < s->count ? 0 : base + blocks, ctx->d_ticket, max_norm, eps, norm, scale ? factor : nullptr,
                                ctx->d_status));
    base += blocks;
    ++launches;
  } while (next < s->count);
  if (!scale) return TWA_OK;
  next = launches == 1 ? next : 0;
  flat = 0;
  do {
    if (launches > 1) next = clip_fill(s, next, &flat, &t);       // else the table is still there
    TWA_CUDA_OK(ctx, twa_launch(ctx->stream, clip_scale_kernel<N>, clip_blocks(ctx, t.chunk[t.count]), CLIP_THREADS, 0, t, factor,
                                out, out_dtype));
  } while (next < s->count);
  return TWA_OK;
}

int clip_any(twa_ctx* ctx, const twa_tensors* s, float max_norm, float eps, bool scale, void* out, int out_dtype, float* norm,
             void* ws, size_t ws_bytes) {
  if (!ws || ws_bytes < twa_grad_norm_workspace_bytes(s->count)) return TWA_ERR_WORKSPACE;
  if (twa_misaligned_to(ws, 16)) return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  if (s->count <= CLIP_FEW) return clip_run<CLIP_FEW>(ctx, s, max_norm, eps, scale, out, out_dtype, norm, ws);
  return clip_run<CLIP_TENSORS>(ctx, s, max_norm, eps, scale, out, out_dtype, norm, ws);
}

}  // namespace

extern "C" {

size_t twa_grad_norm_workspace_bytes(int count) {
  if (count < 0 || count > TWA_MAX_TENSORS) return 0;
  const long long launches = count ? twa_ceil_div(count, CLIP_TENSORS) : 1;
  return CLIP_HEAD + sizeof(double) * CLIP_MAX_BLOCKS * launches;
}

int twa_grad_norm(twa_ctx* ctx, const twa_tensors* tensors, float* norm, void* ws, size_t ws_bytes) {
  int rc = clip_check(ctx, tensors);
  if (rc) return rc;
  if (!norm) return TWA_ERR_INVALID_ARG;
  if (twa_misaligned_to(norm, 4)) return TWA_ERR_MISALIGNED;
  return clip_any(ctx, tensors, 1.0f, 0.0f, false, nullptr, TWA_F32, norm, ws, ws_bytes);
}

int twa_clip_gather(twa_ctx* ctx, const twa_tensors* tensors, float max_norm, float eps, void* g, twa_dtype g_dtype, float* norm,
                    void* ws, size_t ws_bytes) {
  int rc = clip_check(ctx, tensors);
  if (rc) return rc;
  if (!norm || !g || !twa_dtype_ok(g_dtype) || !(max_norm > 0.0f) || !(eps >= 0.0f)) return TWA_ERR_INVALID_ARG;
  if (twa_misaligned_to(norm, 4) || twa_misaligned_to(g, twa_dtype_size(g_dtype))) return TWA_ERR_MISALIGNED;
  return clip_any(ctx, tensors, max_norm, eps, true, g, g_dtype, norm, ws, ws_bytes);
}

int twa_clip_grads(twa_ctx* ctx, const twa_tensors* tensors, float max_norm, float eps, float* norm, void* ws, size_t ws_bytes) {
  int rc = clip_check(ctx, tensors);
  if (rc) return rc;
  if (!norm || !(max_norm > 0.0f) || !(eps >= 0.0f)) return TWA_ERR_INVALID_ARG;
  if (twa_misaligned_to(norm, 4)) return TWA_ERR_MISALIGNED;
  return clip_any(ctx, tensors, max_norm, eps, true, nullptr, TWA_F32, norm, ws, ws_bytes);
}

}  // extern "C"
