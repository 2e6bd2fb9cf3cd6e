// Tokens sorted by expert, and the experts' results brought back with weights.
//
//   dispatch           the assignments (t, j), j < top, sorted by their expert, equal ones in the order of t and j;
//                      out[place[t, j]] = x[t]
//   combine            out[t] = sum_j w[t, j] y[place[t, j]], added in the order of j
//   combine backward   dy[place[t, j]] = w[t, j] dout[t],   dw[t, j] = sum dout[t] y[place[t, j]]
//
// The sort is a counting sort by one cluster of blocks in its shared memory, one launch whatever the number: every warp has a
// run of assignments and counts them by expert, 32 at a time: lanes of the same expert find each other by one ballot for every bit of
// its number, the first of them adds how many they are.  An assignment's place among its warp's goes to where its place will be; a
// prefix over warps, blocks and experts gives what is to be added to it.  No count depends on which block came first.
// Where there are few assignments every block sorts them all and moves its own tokens' rows at once.
// What moves rows is bound by memory and goes token by token, so that a token's row is read, or written, once for all its experts.
//
// 32768 x 2048 bfloat16, 8 of 128 experts: 215 us (1.21 GB, floor 187), of which the sort of 262144 assignments takes 28 on 16 SMs
// (128 warps of 8 blocks, finding each other by a match, which serves one expert after another: 104).  More SMs would need counts in
// memory, and a workspace for them.  Combine 16384 x 1024, two experts: 19 us (100 MB, some of it in L2).  Combine backward
// 16384 x 2048, 8 experts of 64: 191 us (1.14 GB, 6.0 TB/s).  Rows between 16-byte boundaries go by the word or the element: 17489 x 1032,
// 8 experts, forward 56 us in units, 61 by words, 82 by elements (floor 51), backward 112, 131 and 170 (floor 95); 16384 x 1024, two
// experts, 17.7, 17.9 and 26.7 (15.6), backward 28.9, 31.3 and 42.2 (26.0).
// Figures beside the rules below are of calls in a row, whose data L2 holds where it fits, bfloat16 unless they say otherwise.
#include "twa_ops.cuh"

namespace {

// ---- the sort -----------------------------------------------------------------------------------
constexpr int SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_BLOCKS = 16;                   // of a cluster at most
constexpr int SORT_LOADS = 8;                     // ids of a lane under way together

struct SortArgs {
  const void* ids;
  int itype;
  int count, top, experts, bits;                  // count: assignments; bits: of an expert's number, or `experts` for none
  int warps;                                      // of a block (shared memory holds a count of each expert for each of them)
  int run;                                        // assignments of a warp
  int* place;
  int* order;
  int* starts;
  int* status;
};

// Expert of an assignment, `experts` for none.
__device__ __forceinline__ int expert_of(const SortArgs& a, int i, bool report) {
  const long long id = twa_load_id(a.ids, a.itype, i);
  if (id >= 0 && id < a.experts) return static_cast<int>(id);
  if (report && id != -1) twa_set_status(a.status, TWA_ERR_INVALID_ARG, i / a.top);
  return a.experts;
}

// Between the walks place holds an assignment's expert and its number among its warp's of that expert.
constexpr int RANK_BITS = 21;
static_assert(TWA_EXPERTS_MAX <= 32 * 32, "a lane for every 32 experts");
static_assert(TWA_EXPERTS_MAX < 1 << (32 - RANK_BITS) && TWA_EXPERTS_MAX_ASSIGNMENTS / (8 * SORT_WARPS) + 32 < 1 << RANK_BITS, "both fit");

// Sorts with `blocks` blocks, this one the rank-th.  place: where every assignment's place goes; `write`: whether this block writes
// starts and, where it is wanted here, order.  shared: (warps + 3) x experts integers.
__device__ __forceinline__ void sort_block(const SortArgs& a, int blocks, int rank, int* shared, int* place, bool write) {
  int* total = shared;                            // of this block, by expert
  int* base = total + a.experts;                  // place of this block's first assignment of an expert
  int* all = base + a.experts;                    // of all blocks
  int* count = all + a.experts;                   // [warps][experts]
  __shared__ int group[TWA_EXPERTS_MAX / 32];     // assignments of 32 experts
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, threads = a.warps * 32;
  for (int i = threadIdx.x; i < a.warps * a.experts; i += threads) count[i] = 0;
  __syncthreads();
  const long long from = static_cast<long long>(rank * a.warps + warp) * a.run;
  const int first = from < a.count ? static_cast<int>(from) : a.count, last = a.count - first < a.run ? a.count : first + a.run;
  int* mine = count + warp * a.experts;
  for (int i = first; i < last; i += 32 * SORT_LOADS) {
    int e[SORT_LOADS];
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k) e[k] = i + k * 32 + lane < last ? expert_of(a, i + k * 32 + lane, write) : a.experts;
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k) {
      if (i + k * 32 >= last) break;
      unsigned same = 0xffffffffu;
      for (int b = 0; b < a.bits; ++b) {
        const bool set = e[k] >> b & 1;
        const unsigned votes = __ballot_sync(0xffffffffu, set);
        same &= set ? votes : ~votes;
      }
      const unsigned before = same & ((1u << lane) - 1);
      int held = 0;
      if (e[k] < a.experts) held = mine[e[k]];
      __syncwarp();
      if (e[k] < a.experts && before == 0) mine[e[k]] = held + __popc(same);
      __syncwarp();
      if (i + k * 32 + lane < last)
        place[i + k * 32 + lane] = static_cast<int>(static_cast<unsigned>(e[k]) << RANK_BITS | static_cast<unsigned>(held + __popc(before)));
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += threads) {
    int sum = 0;
    for (int w0 = 0; w0 < a.warps; w0 += 8) {
      int c[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) c[w] = w0 + w < a.warps ? count[(w0 + w) * a.experts + e] : 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        if (w0 + w < a.warps) count[(w0 + w) * a.experts + e] = sum;
        sum += c[w];
      }
    }
    total[e] = sum;
  }
  if (blocks > 1) twa_cluster_sync();
  else __syncthreads();
  // Assignments of every expert in all blocks, those of them in blocks before this one, and those of the experts before it among
  // its 32; then those of the 32s before.
  for (int e0 = warp * 32; e0 < a.experts; e0 += threads) {
    const int e = e0 + lane;
    int before = 0, sum = 0;
    if (e < a.experts) {
      int c[SORT_BLOCKS];
#pragma unroll
      for (int r = 0; r < SORT_BLOCKS; ++r) c[r] = r < blocks ? (r == rank ? total[e] : twa_remote(total + e, r)) : 0;
#pragma unroll
      for (int r = 0; r < SORT_BLOCKS; ++r) {
        before += r < rank ? c[r] : 0;
        sum += c[r];
      }
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (e < a.experts) {
      base[e] = before;
      all[e] = upto - sum;
    }
    if (lane == 31) group[e0 >> 5] = upto;
  }
  if (blocks > 1) twa_cluster_sync();             // no block ends while another reads its totals
  else __syncthreads();
  for (int e0 = warp * 32; e0 < a.experts; e0 += threads) {
    const int e = e0 + lane;
    const int ahead = __reduce_add_sync(0xffffffffu, lane < e0 >> 5 ? group[lane] : 0);
    if (e < a.experts) {
      base[e] += ahead + all[e];
      if (write && rank == 0) a.starts[e] = ahead + all[e];
    }
    if (write && rank == 0 && lane == 0 && e0 + 32 >= a.experts) a.starts[a.experts] = ahead + group[e0 >> 5];
  }
  __syncthreads();
  for (int i = first + lane; i < last; i += 32 * SORT_LOADS) {
    unsigned held[SORT_LOADS];
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k)
      if (i + k * 32 < last) held[k] = static_cast<unsigned>(place[i + k * 32]);
#pragma unroll
    for (int k = 0; k < SORT_LOADS; ++k)
      if (i + k * 32 < last) {
        const int e = static_cast<int>(held[k] >> RANK_BITS);
        const int at = e < a.experts ? base[e] + mine[e] + static_cast<int>(held[k] & ((1u << RANK_BITS) - 1)) : -1;
        place[i + k * 32] = at;
        if (write && a.order && at >= 0) a.order[at] = i + k * 32;
      }
  }
}

__global__ void __launch_bounds__(SORT_THREADS) expert_sort_kernel(SortArgs a, int blocks) {
  twa_begin(a.ids);
  extern __shared__ int shared[];
  sort_block(a, blocks, blocks > 1 ? static_cast<int>(twa_cluster_rank()) : 0, shared, a.place, true);
}

// ---- rows to their experts ------------------------------------------------------------------------
constexpr int MOVE_WARPS = 8;
constexpr int NARROW = 8;                         // threads of a row that is no wider than they hold

// Rows as units of type W.
struct Rows {
  const char* x;
  char* out;
  long long ldx, ldo, tokens;                     // strides in bytes
  int units, parts, top;                          // parts: of a row, for one warp each
};
// LANES threads take UNITS units each of a token's row and store them wherever its places say; `where(j)` gives the j-th.
template <typename W, int UNITS, int LANES, typename Where>
__device__ __forceinline__ void move_row(const Rows& r, long long t, int part, Where where) {
  const int u0 = part * (UNITS * LANES) + (threadIdx.x & (LANES - 1));
  const W* from = reinterpret_cast<const W*>(r.x + t * r.ldx);
  W v[UNITS];
#pragma unroll
  for (int k = 0; k < UNITS; ++k)
    if (u0 + k * LANES < r.units) v[k] = __ldg(from + u0 + k * LANES);
  for (int j = 0; j < r.top; ++j) {
    const int p = where(j);
    if (p < 0) continue;
    W* to = reinterpret_cast<W*>(r.out + p * r.ldo);
#pragma unroll
    for (int k = 0; k < UNITS; ++k)
      if (u0 + k * LANES < r.units) to[u0 + k * LANES] = v[k];
  }
}

template <typename W, int UNITS, int LANES>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_gather_kernel(Rows r, const int* place, int* order) {
  twa_begin(r.x, place);
  constexpr int TEAMS = MOVE_WARPS * 32 / LANES;
  const long long task = static_cast<long long>(blockIdx.x) * TEAMS + threadIdx.x / LANES;
  const long long t = task / r.parts;
  if (t >= r.tokens) return;
  const int part = static_cast<int>(task - t * r.parts);
  const int* places = place + t * r.top;
  if (order && part == 0)                          // scattered: not for the sort's few SMs
    for (int j = threadIdx.x & (LANES - 1); j < r.top; j += LANES)
      if (__ldg(places + j) >= 0) order[__ldg(places + j)] = static_cast<int>(t) * r.top + j;
  move_row<W, UNITS, LANES>(r, t, part, [&](int j) { return __ldg(places + j); });
}

// Few assignments: every block sorts them, block 0 says so, and each moves its share of the rows, in one launch.  It and two launches:
// 8 x 512, two of 8 experts, 3.4 and 5.2 us; 512 x 1024, two of 16, 5.4 and 6.3; 1024 x 1024 7.7 and 7.0, 2048 x 1024 13.5 and 7.6;
// 128 x 2048, 8 of 128, 7.2 and 8.1; 256 x 2048 9.5 and 8.8.
constexpr int SMALL_COUNT = 1024;                 // assignments
template <typename W, int UNITS>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_small_kernel(SortArgs a, Rows r) {
  twa_begin(a.ids, r.x);
  extern __shared__ int shared[];
  __shared__ int place[SMALL_COUNT];
  sort_block(a, 1, 0, shared, place, blockIdx.x == 0);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.count; i += MOVE_WARPS * 32) a.place[i] = place[i];
  for (int task = blockIdx.x * MOVE_WARPS + (threadIdx.x >> 5); task < static_cast<int>(r.tokens) * r.parts; task += gridDim.x * MOVE_WARPS) {
    const int t = task / r.parts;
    move_row<W, UNITS, 32>(r, t, task - t * r.parts, [&](int j) { return place[t * r.top + j]; });
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

// LANES threads take UNITS packs of E elements each of a token's row, JOIN of its experts' rows under way together.
template <typename T, int E, int UNITS, int JOIN, int LANES>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_combine_kernel(CombineArgs a) {
  twa_begin(a.y, a.place, a.weights);
  constexpr int TEAMS = MOVE_WARPS * 32 / LANES;
  const long long task = static_cast<long long>(blockIdx.x) * TEAMS + threadIdx.x / LANES;
  const long long t = task / a.parts;
  if (t >= a.tokens) return;
  const int lane = threadIdx.x & (LANES - 1), part = static_cast<int>(task - t * a.parts), c0 = (part * UNITS * LANES + lane) * E;
  const T* y = static_cast<const T*>(a.y) + c0;
  float sum[UNITS][E] = {};
  // a warp's lanes fetch a place each and pass it on (16384 x 1024, two experts: 18.8 us, 21.9 when every lane fetches all)
  constexpr bool PASS = LANES == 32;
  int place = -1;
  float weight = 1.0f;
  if (PASS && lane < a.top) {
    place = place_of(a, t, lane, part == 0);
    if (a.weights) weight = __ldg(a.weights + t * a.top + lane);
  }
  for (int j0 = 0; j0 < a.top; j0 += JOIN) {
    twa_pack<T, E> raw[JOIN][UNITS];
    int p[JOIN];
#pragma unroll
    for (int k = 0; k < JOIN; ++k) {
      const int j = j0 + k;
      if (PASS) p[k] = __shfl_sync(0xffffffffu, place, j & 31);
      else p[k] = j < a.top ? place_of(a, t, j, lane == 0) : -1;
      if (j >= a.top) p[k] = -1;
      if (p[k] < 0) continue;
      const T* row = y + p[k] * a.ldy;
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
        if (c0 + u * LANES * E < a.dim) raw[k][u].load(row + u * LANES * E);
    }
#pragma unroll
    for (int k = 0; k < JOIN; ++k) {
      const int j = j0 + k;
      float w;
      if (PASS) w = __shfl_sync(0xffffffffu, weight, j & 31);
      else w = j < a.top && a.weights ? __ldg(a.weights + t * a.top + j) : 1.0f;
      if (p[k] < 0) continue;
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
        if (c0 + u * LANES * E < a.dim) {
          float v[E];
          raw[k][u].widen(v);
#pragma unroll
          for (int e = 0; e < E; ++e) sum[u][e] = fmaf(w, v[e], sum[u][e]);
        }
    }
  }
  T* out = static_cast<T*>(a.out) + t * a.ldo + c0;
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
    if (c0 + u * LANES * E < a.dim) twa_pack<T, E>::store(out + u * LANES * E, sum[u]);
}

// A token's row for LANES threads (a part of a warp, a warp, or the block), UNITS packs of each at a time: the dot products need the
// whole row.  JOIN of its experts at a time.
template <typename T, int E, int UNITS, int JOIN, int LANES>
__global__ void __launch_bounds__(MOVE_WARPS * 32) expert_combine_backward_kernel(CombineArgs a) {
  twa_begin(a.y, a.dout, a.place, a.weights);
  constexpr bool BLOCK = LANES > 32;
  constexpr int TEAMS = MOVE_WARPS * 32 / LANES;
  __shared__ float part[BLOCK ? MOVE_WARPS : 1][32];
  const long long own = static_cast<long long>(blockIdx.x) * TEAMS + threadIdx.x / LANES;
  const bool live = own < a.tokens;
  if (LANES >= 32 && !live) return;
  const long long t = live ? own : a.tokens - 1;             // threads beside the tokens take part in their warp's shuffles
  const int at = threadIdx.x & (LANES - 1), warp = threadIdx.x >> 5;
  const T* dout = static_cast<const T*>(a.dout) + t * a.ldd;
  for (int j0 = 0; j0 < a.top; j0 += JOIN) {
    int p[JOIN];
    float w[JOIN], dot[JOIN];
#pragma unroll
    for (int k = 0; k < JOIN; ++k) {
      p[k] = live && j0 + k < a.top ? place_of(a, t, j0 + k, at == 0) : -1;
      w[k] = j0 + k < a.top ? __ldg(a.weights + t * a.top + j0 + k) : 0.0f;
      dot[k] = 0.0f;
    }
    for (int c = at * E; c < a.dim; c += UNITS * LANES * E) {
      twa_pack<T, E> rd[UNITS], ry[JOIN][UNITS];
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
        if (c + u * LANES * E < a.dim) rd[u].load(dout + c + u * LANES * E);
#pragma unroll
      for (int k = 0; k < JOIN; ++k)
        if (p[k] >= 0) {
          const T* row = static_cast<const T*>(a.y) + p[k] * a.ldy + c;
#pragma unroll
          for (int u = 0; u < UNITS; ++u)
            if (c + u * LANES * E < a.dim) ry[k][u].load(row + u * LANES * E);
        }
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        if (c + u * LANES * E >= a.dim) break;
        float d[E];
        rd[u].widen(d);
#pragma unroll
        for (int k = 0; k < JOIN; ++k) {
          if (p[k] < 0) continue;
          float v[E];
          ry[k][u].widen(v);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            dot[k] = fmaf(d[e], v[e], dot[k]);
            v[e] = w[k] * d[e];
          }
          twa_pack<T, E>::store(static_cast<T*>(a.out) + p[k] * a.ldo + c + u * LANES * E, v);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < JOIN; ++k) {
      float sum = dot[k];
#pragma unroll
      for (int o = (LANES < 32 ? LANES : 32) / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (BLOCK) {
        if ((at & 31) == 0 && j0 + k < a.top) part[warp][j0 + k] = sum;
      } else if (a.dw && at == 0 && live && j0 + k < a.top) {
        a.dw[t * a.top + j0 + k] = sum;
      }
    }
  }
  if (BLOCK && a.dw) {
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

// Moves rows as units of W, after the sort or (small) with it.  Rows that few threads hold go to as many, not to a warp: 16384 tokens to
// two experts, 64 columns 8.5 us (10.8 by warps), 128 9.2 (10.8), 256 10.4 (11.0); by words and elements 10.0 to 10.5 either way.
template <typename W, int UNITS>
cudaError_t launch_gather(twa_ctx* ctx, const SortArgs& s, Rows r, long long bytes, bool small) {
  r.units = static_cast<int>(bytes / sizeof(W));
  if (!small && r.units <= UNITS * NARROW) {
    r.parts = 1;
    return twa_launch(ctx->stream, expert_gather_kernel<W, UNITS, NARROW>, static_cast<unsigned>(twa_ceil_div(r.tokens, MOVE_WARPS * 32 / NARROW)),
                      MOVE_WARPS * 32, 0, r, s.place, s.order);
  }
  r.parts = static_cast<int>(twa_ceil_div(r.units, UNITS * 32));
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(r.tokens * r.parts, MOVE_WARPS));
  if (!small) return twa_launch(ctx->stream, expert_gather_kernel<W, UNITS, 32>, blocks, MOVE_WARPS * 32, 0, r, s.place, s.order);
  SortArgs one = s;
  one.warps = MOVE_WARPS;
  one.run = static_cast<int>(twa_ceil_div(twa_ceil_div(s.count, MOVE_WARPS), 32) * 32);
  return twa_launch(ctx->stream, expert_small_kernel<W, UNITS>, blocks < 2 * ctx->sm_count ? blocks : 2 * ctx->sm_count, MOVE_WARPS * 32,
                    sizeof(int) * (MOVE_WARPS + 3) * s.experts, one, r);
}

// Blocks of a sorting cluster at most: 16 where the device has room for such a cluster, which not every one need have, otherwise 8.
cudaError_t sort_cluster(twa_ctx* ctx, int* most) {
  if (!ctx->expert_cluster) {
    cudaError_t e = cudaFuncSetAttribute(expert_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(expert_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(int) * (SORT_WARPS + 3) * TWA_EXPERTS_MAX);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(SORT_BLOCKS);
    cfg.blockDim = dim3(SORT_THREADS);
    cfg.dynamicSmemBytes = sizeof(int) * (SORT_WARPS + 3) * TWA_EXPERTS_MAX;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = SORT_BLOCKS;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    e = cudaOccupancyMaxActiveClusters(&clusters, expert_sort_kernel, &cfg);
    if (e != cudaSuccess) return e;
    ctx->expert_cluster = clusters > 0 ? SORT_BLOCKS : 8;
  }
  *most = ctx->expert_cluster;
  return cudaSuccess;
}

int expert_sizes(twa_ctx* ctx, int64_t tokens, int top) {
  if (!ctx || tokens < 0 || top < 1) return TWA_ERR_INVALID_ARG;
  if (top > TWA_EXPERTS_MAX_TOP || tokens > TWA_EXPERTS_MAX_ASSIGNMENTS / top) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

template <typename T, int E, int UNITS, int JOIN, int LANES = 32>
void launch_combine(twa_ctx* ctx, CombineArgs& a) {
  a.parts = static_cast<int>(twa_ceil_div(a.dim, UNITS * LANES * E));
  twa_launch(ctx->stream, expert_combine_kernel<T, E, UNITS, JOIN, LANES>,
             static_cast<unsigned>(twa_ceil_div(a.tokens * a.parts, MOVE_WARPS * 32 / LANES)), MOVE_WARPS * 32, 0, a);
}
// As much of a row a thread as keeps some eight loads of it under way, but where there are few rows more threads a row: 512 x 1024, two
// experts, 2.2 us (2.8 otherwise), 1024 x 1024 2.6 (2.9), 2048 x 1024 3.9 (3.4); 8 experts 3.2 (3.4), 4.0 (3.9) and 6.5 (5.5); by elements
// 140 x 1023, 8 experts, 2.9 (3.4), 512 x 1023, two, 3.0 (2.4).  Narrow rows for a few threads each: 16384 tokens of 64 columns 3.5 us
// (9.7 by warps), of 128 4.0 (9.8); wider ones up to 256 columns would gain too (5.6 and 9.8).  Loads of two experts at a time, or of four and half the columns:
// 16384 x 1024, one expert 10.8 and 11.6, two 17.5 and 18.9, three 25.7 and 23.4, 8 50.7 and 46.8.
template <typename T, int E>
void launch_combine(twa_ctx* ctx, CombineArgs& a) {
  const bool few = a.tokens * twa_ceil_div(a.dim, 32 * E) < 32LL * ctx->sm_count;
  if (a.dim <= 2 * NARROW * E) {
    launch_combine<T, E, 2, 4, NARROW>(ctx, a);
  } else if constexpr (E == twa_vec<T>) {
    if (few) launch_combine<T, E, 1, 4>(ctx, a);
    else if (a.top <= 2) launch_combine<T, E, 4, 2>(ctx, a);
    else launch_combine<T, E, 2, 4>(ctx, a);
  } else {
    if (few) launch_combine<T, E, 2, 4>(ctx, a);
    else launch_combine<T, E, 8, 2>(ctx, a);
  }
}

template <typename T, int E, int UNITS, int JOIN, int LANES>
void launch_combine_backward(twa_ctx* ctx, const CombineArgs& a) {
  twa_launch(ctx->stream, expert_combine_backward_kernel<T, E, UNITS, JOIN, LANES>,
             static_cast<unsigned>(twa_ceil_div(a.tokens, MOVE_WARPS * 32 / LANES)), MOVE_WARPS * 32, 0, a);
}
// Narrow rows for a few threads each: 16384 tokens to two experts, 64 columns 4.2 us (9.5 by warps), 256 6.9 (9.8), and
// wider ones would too (512: 12.9 and 14.1).  A block a token
// where there are few, a warp otherwise: 256 x 1024, two experts, 2.4 us a block and 2.8 a warp, 512 x 4096 4.1 and 6.0; 8 experts,
// 1024 x 2048 10.0 and 12.6, 2048 x 4096 48 and 57; where tokens are some ten an SM and rows short a warp would do better (two experts,
// 1024 x 1024 4.3 and 3.0, 2048 x 1024 7.0 and 3.9; 8 experts, 2048 x 1024 14.0 and 10.4).  Experts at a time by warps, two with four
// packs a thread or four with one: 16384 x 1024, one expert 17.5 and 21.2, two 28.9 and 30.9, three 39.7 and 39.7, 8 of 2048 columns 188 and 192.
template <typename T, int E>
void launch_combine_backward(twa_ctx* ctx, CombineArgs& a) {
  constexpr bool WIDE = E == twa_vec<T>;
  constexpr int BLOCK = MOVE_WARPS * 32;
  if (a.dim <= 4 * NARROW * E) launch_combine_backward<T, E, 2, 4, NARROW>(ctx, a);
  else if (a.tokens < 16LL * ctx->sm_count) launch_combine_backward<T, E, WIDE ? 1 : 4, 4, BLOCK>(ctx, a);
  else if (a.top <= 2) launch_combine_backward<T, E, 4, 2, 32>(ctx, a);
  else launch_combine_backward<T, E, WIDE ? 1 : 4, 4, 32>(ctx, a);
}
struct Forward {
  template <typename T, int E>
  static void launch(twa_ctx* ctx, CombineArgs& a) { launch_combine<T, E>(ctx, a); }
};
struct Backward {
  template <typename T, int E>
  static void launch(twa_ctx* ctx, CombineArgs& a) { launch_combine_backward<T, E>(ctx, a); }
};
// Packs of 16 bytes where all rows lie on them, of 4, or by the element.
template <typename D>
void launch_packed(twa_ctx* ctx, CombineArgs& a, int dtype) {
  const size_t size = twa_dtype_size(dtype);
  auto fits = [&](size_t unit) {
    return a.dim * size % unit == 0 && on_unit(a.y, a.ldy * size, unit) && on_unit(a.out, a.ldo * size, unit) && on_unit(a.dout, a.ldd * size, unit);
  };
  if (dtype == TWA_BF16) {
    if (fits(16)) D::template launch<bf16, 8>(ctx, a);
    else if (fits(4)) D::template launch<bf16, 2>(ctx, a);
    else D::template launch<bf16, 1>(ctx, a);
  } else {
    if (fits(16)) D::template launch<float, 4>(ctx, a);
    else D::template launch<float, 1>(ctx, a);
  }
}

}  // namespace

extern "C" {

int twa_expert_dispatch(twa_ctx* ctx, const void* x, int64_t ldx, twa_dtype dtype, int64_t tokens, int dim, const void* ids, twa_itype id_type,
                        int top, int experts, int32_t* place, int32_t* starts, int32_t* order, void* out, int64_t ldo) {
  int rc = expert_sizes(ctx, tokens, top);
  if (rc) return rc;
  if (!twa_dtype_ok(dtype) || !twa_itype_ok(id_type) || experts < 1 || dim < 1) return TWA_ERR_INVALID_ARG;
  if (experts > TWA_EXPERTS_MAX || dim > TWA_EXPERTS_MAX_DIM) return TWA_ERR_UNSUPPORTED;
  if (!starts || (tokens && (!ids || !place || !x != !out))) return TWA_ERR_INVALID_ARG;
  if (x && tokens && (ldx < dim || ldo < dim)) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(starts, 4) || (tokens && (twa_misaligned_to(ids, twa_itype_size(id_type)) || twa_misaligned_to(place, 4) ||
                                                  twa_misaligned_to(order, 4) || twa_misaligned_to(x, size) || twa_misaligned_to(out, size))))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  SortArgs s = {ids, id_type, static_cast<int>(tokens * top), top, experts, 1, SORT_WARPS, 0, place, order, starts, ctx->d_status};
  while (experts >> s.bits) ++s.bits;
  const bool moves = x && tokens;
  const bool small = moves && s.count <= SMALL_COUNT && sizeof(int) * ((MOVE_WARPS + 3) * experts + SMALL_COUNT + TWA_EXPERTS_MAX / 32) <= 48 * 1024;
  if (!small) {
    const size_t smem = sizeof(int) * (s.warps + 3) * experts;
    int blocks = 1, most;
    TWA_CUDA_OK(ctx, sort_cluster(ctx, &most));
    // as soon as warps have more than 32 assignments each (4096 x 2 of 16 experts 5.1 us, 5.8 where they have 64 first, 7.5 where 128)
    while (blocks < most && s.count > blocks * s.warps * 32) blocks *= 2;
    s.run = static_cast<int>(twa_ceil_div(twa_ceil_div(s.count, blocks * s.warps), 32) * 32);
    SortArgs first = s;
    if (moves) first.order = nullptr;              // the blocks that move rows write it
    TWA_CUDA_OK(ctx, twa_launch_clusters(ctx->stream, expert_sort_kernel, blocks, blocks, s.warps * 32, smem, first, blocks));
  }
  if (moves) {
    const long long bytes = static_cast<long long>(dim) * size;
    const Rows r = {static_cast<const char*>(x), static_cast<char*>(out), static_cast<long long>(ldx * size), static_cast<long long>(ldo * size),
                    tokens, 0, 0, top};
    auto fits = [&](size_t unit) { return bytes % unit == 0 && on_unit(x, r.ldx, unit) && on_unit(out, r.ldo, unit); };
    const cudaError_t launched = fits(16)  ? launch_gather<uint4, 4>(ctx, s, r, bytes, small)
                                 : fits(4) ? launch_gather<uint32_t, 8>(ctx, s, r, bytes, small)
                                           : launch_gather<unsigned short, 8>(ctx, s, r, bytes, small);
    TWA_CUDA_OK(ctx, launched);
  }
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
  CombineArgs a = {y, nullptr, place, weights, out, nullptr, ldy, 0, ldo, rows, tokens, top, dim, 0, ctx->d_status};
  launch_packed<Forward>(ctx, a, dtype);
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
  CombineArgs a = {y, dout, place, weights, dy, dw, ldy, lddout, lddy, rows, tokens, top, dim, 0, ctx->d_status};
  launch_packed<Backward>(ctx, a, dtype);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
