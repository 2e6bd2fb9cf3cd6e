// Embedding lookup with scaling, and the gradient of the table.
//
//   forward    out[t] = scale * table[ids[t]]
//   backward   dtable[v] = scale * sum over t with ids[t] == v of dout[t], in the order of t
//
// Forward is a gather: every row of the output is written once, a row of the table read from memory or from L2.
// Backward sorts (id, position) by id with a stable radix sort, so that equal ids lie side by side in the order of
// their positions, and adds the rows of each id in that order: the sum does not depend on which block came first, and
// a frequent token costs no conflicting atomics.  The sorted list is cut into runs of EMB_RUN entries whatever the
// ids are (a run is one block's work, so a frequent token is shared by many blocks); an id that crosses the end of a
// run leaves a float32 partial sum per run, and a last kernel adds those in run order.  Rows of the table that no token
// names are set to zero by a kernel that needs only the ids' bitmap.
#include "twa_ops.cuh"

namespace {

constexpr int SORT_THREADS = 256, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_KEYS = 8;                               // keys of a thread
constexpr int SORT_TILE = SORT_THREADS * SORT_KEYS;        // keys of a block
constexpr int SORT_MAX_BITS = 9, SORT_BINS = 1 << SORT_MAX_BITS;
constexpr int EMB_RUN = 32;                                // sorted entries a block adds up

// E elements of any pairing of the two types; E = 8 wants both addresses on 16 bytes, E = 1 nothing.
template <typename T, int E>
__device__ __forceinline__ void load_row(const T* p, float* v) {
  if constexpr (E == 1) v[0] = twa_to_float(p[0]);
  else
#pragma unroll
    for (int i = 0; i < E; i += twa_vec<T>) {
      twa_pack<T, twa_vec<T>> q;
      q.load(p + i);
      q.widen(v + i);
    }
}
template <typename T, int E>
__device__ __forceinline__ void store_row(T* p, const float* v) {
  if constexpr (E == 1) p[0] = twa_from_float<T>(v[0]);
  else
#pragma unroll
    for (int i = 0; i < E; i += twa_vec<T>) twa_pack<T, twa_vec<T>>::store(p + i, v + i);
}

// ---- forward -------------------------------------------------------------------------------------
// A warp takes FWD_UNITS x 32 units of E elements of one row.
constexpr int FWD_UNITS = 4, FWD_WARPS = 4;

template <typename TT, typename TO, int E>
__global__ void embedding_kernel(const TT* __restrict__ table, long long ldt, int vocab, const void* __restrict__ ids, int itype,
                                 long long tokens, int dim, float scale, TO* __restrict__ out, long long ldo, int parts,
                                 int* status) {
  const long long task = static_cast<long long>(blockIdx.x) * FWD_WARPS + (threadIdx.x >> 5);
  const long long t = task / parts;
  if (t >= tokens) return;
  const int part = static_cast<int>(task - t * parts);
  const long long id = twa_load_id(ids, itype, t);
  const bool good = id >= 0 && id < vocab;
  if (!good && part == 0 && (threadIdx.x & 31) == 0) twa_set_status(status, TWA_ERR_INVALID_ARG, static_cast<int>(t));
  const int c0 = (part * FWD_UNITS * 32 + (threadIdx.x & 31)) * E;
  float v[FWD_UNITS][E];
#pragma unroll
  for (int k = 0; k < FWD_UNITS; ++k) {
    const int c = c0 + k * 32 * E;
#pragma unroll
    for (int e = 0; e < E; ++e) v[k][e] = 0.0f;
    if (good && c < dim) load_row<TT, E>(table + id * ldt + c, v[k]);
  }
#pragma unroll
  for (int k = 0; k < FWD_UNITS; ++k) {
    const int c = c0 + k * 32 * E;
#pragma unroll
    for (int e = 0; e < E; ++e) v[k][e] *= scale;
    if (c < dim) store_row<TO, E>(out + t * ldo + c, v[k]);
  }
}

// ---- the sort --------------------------------------------------------------------------------------
// Layout of the workspace.
struct EmbSpace {
  uint32_t *key[2], *pos[2];      // tokens each
  int* hist[2];                   // [tiles][SORT_BINS]
  uint32_t* used;                 // bitmap of the ids that occur
  float* partial;                 // [runs][2][dim]
  size_t bytes;
};
EmbSpace emb_space(void* ws, long long tokens, long long vocab, long long dim) {
  EmbSpace s;
  char* p = static_cast<char*>(ws);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* r = p ? p + at : nullptr;
    at += twa_round256(bytes);
    return r;
  };
  const long long tiles = twa_ceil_div(tokens, SORT_TILE), runs = twa_ceil_div(tokens, EMB_RUN);
  // cleared together at the start of a call: bitmap, then the two sets of counts
  s.used = reinterpret_cast<uint32_t*>(take(twa_ceil_div(vocab, 32) * 4));
  for (int i = 0; i < 2; ++i) s.hist[i] = reinterpret_cast<int*>(take(sizeof(int) * SORT_BINS * tiles));
  for (int i = 0; i < 2; ++i) s.key[i] = reinterpret_cast<uint32_t*>(take(4 * tokens));
  for (int i = 0; i < 2; ++i) s.pos[i] = reinterpret_cast<uint32_t*>(take(4 * tokens));
  s.partial = reinterpret_cast<float*>(take(sizeof(float) * 2 * dim * runs));
  s.bytes = at;
  return s;
}

// Sort key of a token: its id, or `vocab` (after every id) where it contributes nothing.
__device__ __forceinline__ uint32_t emb_key(const void* ids, int itype, long long t, int vocab, long long padding, int* status) {
  const long long id = twa_load_id(ids, itype, t);
  if (id >= 0 && id < vocab) return id == padding ? static_cast<uint32_t>(vocab) : static_cast<uint32_t>(id);
  if (status) twa_set_status(status, TWA_ERR_INVALID_ARG, static_cast<int>(t));
  return static_cast<uint32_t>(vocab);
}

// Counts of the first digit per tile; marks the ids that occur.
__global__ void emb_count_kernel(const void* __restrict__ ids, int itype, int tokens, int vocab, long long padding, int bits,
                                 uint32_t* used, int* __restrict__ hist, int* status) {
  __shared__ int count[SORT_BINS];
  const int bins = 1 << bits;
  for (int d = threadIdx.x; d < bins; d += SORT_THREADS) count[d] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < SORT_TILE; i += SORT_THREADS) {
    const long long t = static_cast<long long>(blockIdx.x) * SORT_TILE + i;
    if (t >= tokens) break;
    const uint32_t key = emb_key(ids, itype, t, vocab, padding, status);
    atomicAdd(&count[key & (bins - 1)], 1);
    if (key < static_cast<uint32_t>(vocab)) atomicOr(&used[key >> 5], 1u << (key & 31));
  }
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += SORT_THREADS) hist[blockIdx.x * SORT_BINS + d] = count[d];
}

// One pass of the radix sort over the digit at `shift`: stable, a tile per block.  key_in == null: the keys are the ids'.
// Counts the next digit of every key in the tile that the key moves to (hist_next, cleared; integer sums).
__global__ void emb_scatter_kernel(const void* __restrict__ ids, int itype, int vocab, long long padding,
                                   const uint32_t* __restrict__ key_in, const uint32_t* __restrict__ pos_in, int tokens,
                                   int shift, int bits, const int* __restrict__ hist, int* __restrict__ hist_next,
                                   uint32_t* __restrict__ key_out, uint32_t* __restrict__ pos_out) {
  __shared__ int count[SORT_WARPS][SORT_BINS];
  __shared__ int base[SORT_BINS];
  __shared__ int warp_total[SORT_WARPS];
  const int bins = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tile = blockIdx.x, tiles = gridDim.x;
  for (int d = threadIdx.x; d < SORT_WARPS * SORT_BINS; d += SORT_THREADS) (&count[0][0])[d] = 0;
  __syncthreads();
  // rank of every key among the equal digits of its warp, in the order of the keys
  uint32_t key[SORT_KEYS], pos[SORT_KEYS];
  int rank[SORT_KEYS];
  const int t0 = tile * SORT_TILE + warp * 32 * SORT_KEYS + lane;
#pragma unroll
  for (int k = 0; k < SORT_KEYS; ++k) {
    const int t = t0 + k * 32;
    key[k] = 0;
    pos[k] = t;
    if (t < tokens) {
      key[k] = key_in ? key_in[t] : emb_key(ids, itype, t, vocab, padding, nullptr);
      if (key_in) pos[k] = pos_in[t];
    }
  }
#pragma unroll
  for (int k = 0; k < SORT_KEYS; ++k) {
    const bool in = t0 + k * 32 < tokens;
    const int d = (key[k] >> shift) & (bins - 1);
    const unsigned same = __match_any_sync(0xffffffffu, in ? d : -1);
    const int before = __popc(same & ((1u << lane) - 1));
    rank[k] = in ? count[warp][d] + before : 0;
    __syncwarp();
    if (in && before == 0) count[warp][d] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // where the tile's keys of each digit begin: keys of smaller digits, then of the same digit in earlier tiles, then warps
  int carry = 0;
  for (int d0 = 0; d0 < bins; d0 += SORT_THREADS) {
    const int d = d0 + threadIdx.x;
    int all = 0, earlier = 0;
    if (d < bins)
      for (int k = 0; k < tiles; ++k) {
        const int c = __ldg(hist + k * SORT_BINS + d);
        if (k < tile) earlier += c;
        all += c;
      }
    int sum = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 31) warp_total[warp] = sum;
    __syncthreads();
    int below = carry;
    for (int k = 0; k < SORT_WARPS; ++k) {
      if (k < warp) below += warp_total[k];
      carry += warp_total[k];
    }
    if (d < bins) base[d] = below + sum - all + earlier;
    __syncthreads();
  }
  for (int d = threadIdx.x; d < bins; d += SORT_THREADS) {
    int at = base[d];
    for (int k = 0; k < SORT_WARPS; ++k) {
      const int c = count[k][d];
      count[k][d] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < SORT_KEYS; ++k) {
    if (t0 + k * 32 >= tokens) continue;
    const int to = count[warp][(key[k] >> shift) & (bins - 1)] + rank[k];
    key_out[to] = key[k];
    pos_out[to] = pos[k];
    if (hist_next) atomicAdd(&hist_next[to / SORT_TILE * SORT_BINS + ((key[k] >> (shift + bits)) & (bins - 1))], 1);
  }
}

// ---- zero rows, sums, joins ------------------------------------------------------------------------
template <typename T, int E>
__global__ void emb_zero_kernel(const uint32_t* __restrict__ used, int vocab, int dim, T* __restrict__ dtable, long long ldg) {
  float zero[E];
#pragma unroll
  for (int e = 0; e < E; ++e) zero[e] = 0.0f;
  for (long long v = blockIdx.x; v < vocab; v += gridDim.x) {
    if (__ldg(used + (v >> 5)) >> (v & 31) & 1) continue;
    for (int c = threadIdx.x * E; c < dim; c += blockDim.x * E) store_row<T, E>(dtable + v * ldg + c, zero);
  }
}

template <typename TG, int E>
__device__ __forceinline__ void emb_write(TG* to, float (&sum)[E], float scale, int accumulate) {
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] *= scale;
  if (accumulate) {
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += twa_to_float(to[e]);
  }
  store_row<TG, E>(to, sum);
}

// Run blockIdx.x of the sorted list, columns of blockIdx.y: the rows of every id in the run are added in order.  An id
// that also lies in the run before, or in the run after, leaves its sum in partial[run][0], or [run][1].
template <typename TD, typename TG, int E>
__global__ void emb_sum_kernel(const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos, int tokens, int vocab, int dim,
                               const TD* __restrict__ dout, long long ldd, float scale, TG* __restrict__ dtable, long long ldg,
                               int accumulate, float* __restrict__ partial) {
  constexpr int AHEAD = 4;
  __shared__ uint32_t k[EMB_RUN + 2], p[EMB_RUN];
  const int first = blockIdx.x * EMB_RUN, n = min(EMB_RUN, tokens - first);
  if (threadIdx.x < EMB_RUN + 2) {
    const int i = first + static_cast<int>(threadIdx.x) - 1;      // one entry before and one after
    k[threadIdx.x] = i >= 0 && i < tokens ? key[i] : 0xffffffffu;
    if (threadIdx.x >= 1 && static_cast<int>(threadIdx.x) <= n) p[threadIdx.x - 1] = pos[i];
  }
  __syncthreads();
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * E;
  if (c >= dim) return;
  float sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0f;
  for (int i0 = 0; i0 < n; i0 += AHEAD) {
    float v[AHEAD][E];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (i0 + j < n && k[i0 + j + 1] < static_cast<uint32_t>(vocab))
        load_row<TD, E>(dout + static_cast<long long>(p[i0 + j]) * ldd + c, v[j]);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = i0 + j;
      if (i >= n) break;
      const uint32_t id = k[i + 1];
      if (id >= static_cast<uint32_t>(vocab)) return;             // the rest contributes nothing
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += v[j][e];
      const bool last = i + 1 == n;
      if (!last && k[i + 2] == id) continue;
      const bool before = k[0] == id, after = last && k[i + 2] == id;
      if (before || after) {
        float* to = partial + (static_cast<long long>(blockIdx.x) * 2 + (before ? 0 : 1)) * dim + c;
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = sum[e];
      } else {
        emb_write<TG, E>(dtable + static_cast<long long>(id) * ldg + c, sum, scale, accumulate);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    }
  }
}

// An id that begins in run blockIdx.x and goes on: its partial sums over the runs, JOIN_WAYS stretches of runs side by side.
constexpr int JOIN_WAYS = 8, JOIN_LANES = 32;
template <typename TG, int E>
__global__ void emb_join_kernel(const uint32_t* __restrict__ key, int tokens, int vocab, int dim, float scale,
                                TG* __restrict__ dtable, long long ldg, int accumulate, const float* __restrict__ partial) {
  __shared__ float part[JOIN_WAYS][JOIN_LANES][E + 1];
  const long long first = static_cast<long long>(blockIdx.x) * EMB_RUN, next = first + EMB_RUN;
  if (next >= tokens) return;
  const uint32_t id = key[next - 1];
  if (id >= static_cast<uint32_t>(vocab) || key[next] != id) return;
  if (first > 0 && key[first - 1] == id) return;                  // it began in an earlier run
  long long low = next, high = tokens;                            // the first entry after the id's
  while (low < high) {
    const long long mid = (low + high) / 2;
    if (key[mid] == id) low = mid + 1;
    else high = mid;
  }
  const int from = blockIdx.x, to = static_cast<int>((low - 1) / EMB_RUN) + 1;    // runs
  const int lane = threadIdx.x % JOIN_LANES, way = threadIdx.x / JOIN_LANES;
  const int each = (to - from + JOIN_WAYS - 1) / JOIN_WAYS;
  const int a = from + way * each, b = min(to, a + each);
  for (int c0 = 0; c0 < dim; c0 += JOIN_LANES * E) {
    const int c = c0 + lane * E;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    if (c < dim)
      for (int r = a; r < b; ++r) {
        const float* src = partial + (static_cast<long long>(r) * 2 + (r == from ? 1 : 0)) * dim + c;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += src[e];
      }
#pragma unroll
    for (int e = 0; e < E; ++e) part[way][lane][e] = sum[e];
    __syncthreads();
    if (way == 0 && c < dim) {
      for (int w = 1; w < JOIN_WAYS; ++w)
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += part[w][lane][e];
      emb_write<TG, E>(dtable + static_cast<long long>(id) * ldg + c, sum, scale, accumulate);
    }
    __syncthreads();
  }
}

bool emb_packs(const void* p, long long ld, size_t size) { return !twa_misaligned_to(p, 16) && (ld * size) % 16 == 0; }

template <typename TT, typename TO>
void launch_embedding(twa_ctx* ctx, bool packs, const void* table, int64_t ldt, int vocab, const void* ids, int itype,
                      int64_t tokens, int dim, float scale, void* out, int64_t ldo) {
  const int parts = static_cast<int>(twa_ceil_div(dim, (packs ? 8 : 1) * 32 * FWD_UNITS));
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(tokens * parts, FWD_WARPS));
  if (packs)
    embedding_kernel<TT, TO, 8><<<blocks, 32 * FWD_WARPS, 0, ctx->stream>>>(static_cast<const TT*>(table), ldt, vocab, ids, itype,
                                                                          tokens, dim, scale, static_cast<TO*>(out), ldo, parts,
                                                                          ctx->d_status);
  else
    embedding_kernel<TT, TO, 1><<<blocks, 32 * FWD_WARPS, 0, ctx->stream>>>(static_cast<const TT*>(table), ldt, vocab, ids, itype,
                                                                          tokens, dim, scale, static_cast<TO*>(out), ldo, parts,
                                                                          ctx->d_status);
}

template <typename TD, typename TG, int E>
void launch_sums(twa_ctx* ctx, const EmbSpace& s, const uint32_t* key, const uint32_t* pos, int tokens, int vocab, int dim,
                 const void* dout, int64_t ldd, float scale, void* dtable, int64_t ldg, int accumulate) {
  TG* g = static_cast<TG*>(dtable);
  if (tokens) {
    const unsigned runs = static_cast<unsigned>(twa_ceil_div(tokens, EMB_RUN));
    const int units = (dim + E - 1) / E, threads = units >= 128 ? 128 : (units < 64 ? 64 : (units + 31) / 32 * 32);
    const dim3 grid(runs, static_cast<unsigned>(twa_ceil_div(units, threads)));
    emb_sum_kernel<TD, TG, E><<<grid, threads, 0, ctx->stream>>>(key, pos, tokens, vocab, dim, static_cast<const TD*>(dout), ldd,
                                                                 scale, g, ldg, accumulate, s.partial);
    if (runs > 1)
      emb_join_kernel<TG, E><<<runs - 1, JOIN_WAYS * JOIN_LANES, 0, ctx->stream>>>(key, tokens, vocab, dim, scale, g, ldg,
                                                                                 accumulate, s.partial);
  }
}

template <typename TD, typename TG>
void launch_sums_any(twa_ctx* ctx, bool packs, const EmbSpace& s, const uint32_t* key, const uint32_t* pos, int tokens, int vocab,
                     int dim, const void* dout, int64_t ldd, float scale, void* dtable, int64_t ldg, int accumulate) {
  if (packs) launch_sums<TD, TG, 8>(ctx, s, key, pos, tokens, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate);
  else launch_sums<TD, TG, 1>(ctx, s, key, pos, tokens, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate);
}

template <typename TG>
void launch_zero(twa_ctx* ctx, bool packs, const uint32_t* used, int vocab, int dim, void* dtable, int64_t ldg) {
  const int blocks = vocab < 8 * ctx->sm_count ? vocab : 8 * ctx->sm_count;
  if (packs) emb_zero_kernel<TG, 8><<<blocks, 256, 0, ctx->stream>>>(used, vocab, dim, static_cast<TG*>(dtable), ldg);
  else emb_zero_kernel<TG, 1><<<blocks, 256, 0, ctx->stream>>>(used, vocab, dim, static_cast<TG*>(dtable), ldg);
}

}  // namespace

extern "C" {

int twa_embedding(twa_ctx* ctx, const void* table, int64_t ldt, twa_dtype t_dtype, int vocab, int dim, const void* ids,
                  twa_itype id_type, int64_t tokens, float scale, void* out, int64_t ldo, twa_dtype out_dtype) {
  if (!ctx || !twa_dtype_ok(t_dtype) || !twa_dtype_ok(out_dtype) || !twa_itype_ok(id_type)) return TWA_ERR_INVALID_ARG;
  if (vocab < 1 || dim < 1 || tokens < 0) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_EMBEDDING_MAX_TOKENS || dim > TWA_EMBEDDING_MAX_DIM) return TWA_ERR_UNSUPPORTED;
  if (tokens == 0) return TWA_OK;
  if (!table || !ids || !out || ldt < dim || ldo < dim) return TWA_ERR_INVALID_ARG;
  const size_t ts = twa_dtype_size(t_dtype), os = twa_dtype_size(out_dtype);
  if (twa_misaligned_to(table, ts) || twa_misaligned_to(out, os) || twa_misaligned_to(ids, twa_itype_size(id_type)))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  const bool packs = dim % 8 == 0 && emb_packs(table, ldt, ts) && emb_packs(out, ldo, os);
  const bool tb = t_dtype == TWA_BF16, ob = out_dtype == TWA_BF16;
  if (tb && ob) launch_embedding<bf16, bf16>(ctx, packs, table, ldt, vocab, ids, id_type, tokens, dim, scale, out, ldo);
  else if (tb) launch_embedding<bf16, float>(ctx, packs, table, ldt, vocab, ids, id_type, tokens, dim, scale, out, ldo);
  else if (ob) launch_embedding<float, bf16>(ctx, packs, table, ldt, vocab, ids, id_type, tokens, dim, scale, out, ldo);
  else launch_embedding<float, float>(ctx, packs, table, ldt, vocab, ids, id_type, tokens, dim, scale, out, ldo);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

size_t twa_embedding_workspace_bytes(int64_t tokens, int vocab, int dim) {
  if (tokens < 0 || tokens > TWA_EMBEDDING_MAX_TOKENS || vocab < 1 || dim < 1 || dim > TWA_EMBEDDING_MAX_DIM) return 0;
  return emb_space(nullptr, tokens, vocab, dim).bytes;
}

int twa_embedding_backward(twa_ctx* ctx, const void* dout, int64_t ldd, twa_dtype d_dtype, const void* ids, twa_itype id_type,
                           int64_t tokens, int vocab, int dim, float scale, int64_t padding_id, void* dtable, int64_t ldg,
                           twa_dtype g_dtype, int accumulate, void* ws, size_t ws_bytes) {
  if (!ctx || !twa_dtype_ok(d_dtype) || !twa_dtype_ok(g_dtype) || !twa_itype_ok(id_type)) return TWA_ERR_INVALID_ARG;
  if (vocab < 1 || dim < 1 || tokens < 0 || accumulate < 0 || accumulate > 1) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_EMBEDDING_MAX_TOKENS || dim > TWA_EMBEDDING_MAX_DIM) return TWA_ERR_UNSUPPORTED;
  if (!dtable || ldg < dim || (tokens && (!dout || !ids || ldd < dim))) return TWA_ERR_INVALID_ARG;
  const size_t ds = twa_dtype_size(d_dtype), gs = twa_dtype_size(g_dtype);
  if (twa_misaligned_to(dout, ds) || twa_misaligned_to(dtable, gs) || twa_misaligned_to(ids, twa_itype_size(id_type)))
    return TWA_ERR_MISALIGNED;
  if (!ws || ws_bytes < twa_embedding_workspace_bytes(tokens, vocab, dim)) return TWA_ERR_WORKSPACE;
  if (twa_misaligned_to(ws, 16)) return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  const EmbSpace s = emb_space(ws, tokens, vocab, dim);
  const int n = static_cast<int>(tokens), tiles = static_cast<int>(twa_ceil_div(tokens, SORT_TILE));
  const bool packs = dim % 8 == 0 && emb_packs(dout, ldd, ds) && emb_packs(dtable, ldg, gs);
  TWA_CUDA_OK(ctx, cudaMemsetAsync(s.used, 0, reinterpret_cast<char*>(s.key[0]) - reinterpret_cast<char*>(s.used), ctx->stream));
  int total_bits = 1;
  while (total_bits < 32 && (static_cast<long long>(vocab) >> total_bits)) ++total_bits;      // keys 0 .. vocab
  const int passes = (total_bits + SORT_MAX_BITS - 1) / SORT_MAX_BITS, bits = (total_bits + passes - 1) / passes;
  int at = 0;
  if (n) {
    emb_count_kernel<<<tiles, SORT_THREADS, 0, ctx->stream>>>(ids, id_type, n, vocab, padding_id, bits, s.used, s.hist[0],
                                                              ctx->d_status);
    for (int p = 0; p < passes; ++p) {
      int* next = p + 1 < passes ? s.hist[(p + 1) & 1] : nullptr;
      if (p >= 1 && next)
        TWA_CUDA_OK(ctx, cudaMemsetAsync(next, 0, sizeof(int) * SORT_BINS * tiles, ctx->stream));
      emb_scatter_kernel<<<tiles, SORT_THREADS, 0, ctx->stream>>>(ids, id_type, vocab, padding_id, p ? s.key[at] : nullptr,
                                                                  p ? s.pos[at] : nullptr, n, p * bits, bits, s.hist[p & 1], next,
                                                                  s.key[at ^ 1], s.pos[at ^ 1]);
      at ^= 1;
    }
    TWA_CUDA_OK(ctx, cudaGetLastError());
  }
  const bool db = d_dtype == TWA_BF16, gb = g_dtype == TWA_BF16;
  if (!accumulate) {
    if (gb) launch_zero<bf16>(ctx, packs, s.used, vocab, dim, dtable, ldg);
    else launch_zero<float>(ctx, packs, s.used, vocab, dim, dtable, ldg);
  }
  const uint32_t *key = s.key[at], *pos = s.pos[at];
  if (db && gb) launch_sums_any<bf16, bf16>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate);
  else if (db) launch_sums_any<bf16, float>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate);
  else if (gb) launch_sums_any<float, bf16>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate);
  else launch_sums_any<float, float>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
