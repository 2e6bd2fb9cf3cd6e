// Embedding lookup with scaling, and the gradient of the table.
//
//   forward    out[t] = scale * table[ids[t]]
//   backward   dtable[v] = scale * sum over t with ids[t] == v of dout[t], in the order of t
//
// Forward is a gather: every row of the output is written once, a row of the table read from memory or from L2.
// Backward sorts (id, position) by id with a stable radix sort, so that equal ids lie side by side in the order of
// their positions, and adds the rows of each id in that order: the sum does not depend on which block came first, and
// a frequent token costs no conflicting atomics.  The sorted list is cut into runs of EMB_RUN entries whatever the
// ids are; a run is one block's work.  An id that goes on into the next run and ends there is added up by the block of
// the run it begins in.  One that covers a run whole (a frequent token) leaves a float32 partial sum in each of its runs,
// and a last kernel adds those in run order.
//
// Most of what a whole table's gradient has to write are the zeros of rows that no token names.  They need the ids'
// bitmap only, which the first, short kernel leaves: the kernels that sort, latency-bound on a few SMs, carry blocks that
// write zeros on the others, and the rest of them go beside the sums.  Up to 16384 ids a cluster of blocks sorts them in
// its shared memory, in one launch; the zeros beside it go to rows whether used or not (the sums come later).
//
// Forward 2048 x 2048 out of a float32 table: 6 us, most of it the call.  Backward 16384 x 2048 bfloat16 into 50272 float32
// rows: 81.7 us for 479 MB, 5.9 TB/s; 26 us the sort with its zeros, 48 the sums with the rest.  Beyond 16384 ids a pass of the
// sort adds the counts of all tiles in each tile, which grows with the square of the ids: 32768 ids 108 us (floor 83), 131072
// 201 (145), 2^20 1266 (720).
#include "twa_ops.cuh"

namespace {

constexpr int SORT_THREADS = 256, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_KEYS = 4;                               // keys of a thread
constexpr int SORT_TILE = SORT_THREADS * SORT_KEYS;        // keys of a block
constexpr int SORT_MAX_BITS = 9, SORT_BINS = 1 << SORT_MAX_BITS;
constexpr int EMB_RUN = 32;                                // sorted entries a block adds up
constexpr int SMALL_THREADS = 512, SMALL_WARPS = SMALL_THREADS / 32, SMALL_TILE = SMALL_THREADS * SORT_KEYS;
constexpr int SMALL_BLOCKS = 8, SMALL_TOKENS = SMALL_BLOCKS * SMALL_TILE;      // of a cluster
constexpr int SMALL_BITS = 8, SMALL_BINS = 1 << SMALL_BITS;
constexpr int SMALL_VOCAB = 1 << 20;                       // ids whose bitmap a block clears
// Zeros of a block: with 16384 x 2048 into 50272 rows and 96 MB beside the sort 88.6 us with 8 KB, 85.2 with 16, 88.1 with 32.
constexpr int FILL_BYTES = 1 << 14;
constexpr int FILL_TEAM = 7;                               // log2 of the threads a row, those of the smallest block that writes zeros
// Zeros written beside a sorting kernel: what its few us have room for.
constexpr long long FILL_BESIDE_SORT = 32LL << 20;

// E elements of any pairing of the two types; E = 8 wants both addresses on 16 bytes, E = 1 nothing.
template <typename T, int E>
__device__ __forceinline__ void load_row(const T* p, float* v) {
  constexpr int N = E == 1 ? 1 : twa_vec<T>;
#pragma unroll
  for (int i = 0; i < E; i += N) {
    twa_pack<T, N> q;
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
template <int E>
constexpr int FWD_UNITS = E == 1 ? 16 : 4;
constexpr int FWD_WARPS = 4;

template <typename TT, typename TO, int E>
__global__ void embedding_kernel(const TT* __restrict__ table, long long ldt, int vocab, const void* __restrict__ ids, int itype,
                                 long long tokens, int dim, float scale, TO* __restrict__ out, long long ldo, int parts,
                                 int* status) {
  twa_begin(table, ids);
  const long long task = static_cast<long long>(blockIdx.x) * FWD_WARPS + (threadIdx.x >> 5);
  const long long t = task / parts;
  if (t >= tokens) return;
  const int part = static_cast<int>(task - t * parts);
  const long long id = twa_load_id(ids, itype, t);
  const bool good = id >= 0 && id < vocab;
  if (!good && part == 0 && (threadIdx.x & 31) == 0) twa_set_status(status, TWA_ERR_INVALID_ARG, static_cast<int>(t));
  const int c0 = (part * FWD_UNITS<E> * 32 + (threadIdx.x & 31)) * E;
  float v[FWD_UNITS<E>][E];
#pragma unroll
  for (int k = 0; k < FWD_UNITS<E>; ++k) {
    const int c = c0 + k * 32 * E;
#pragma unroll
    for (int e = 0; e < E; ++e) v[k][e] = 0.0f;
    if (good && c < dim) load_row<TT, E>(table + id * ldt + c, v[k]);
  }
#pragma unroll
  for (int k = 0; k < FWD_UNITS<E>; ++k) {
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
  twa_begin(ids);
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

// The rows of a table as bytes, for writing zeros; `each` rows a block.
struct EmbFill {
  char* table;
  long long stride;             // bytes between rows
  long long bytes;              // of a row
  const uint32_t* used;         // null: all rows
  int row0, row1, each;         // rows row0 .. row1 - 1
  int size;                     // of an element
  int log_team;                 // log2 of the threads that write a row together, at most FILL_TEAM
};
// Zeros into the unused ones of the block's rows (or all): 16 bytes a store between the ragged ends.  A team takes a row at a time,
// so that a store costs no division and no look at the bitmap.
__device__ __forceinline__ void emb_fill(const EmbFill& f, int block) {
  const int r0 = f.row0 + block * f.each, rows = min(f.each, f.row1 - r0);      // none for a cluster's spare blocks
  const int step = 1 << f.log_team, team = threadIdx.x >> f.log_team, t = threadIdx.x & (step - 1);
  for (int v = r0 + team; v < r0 + rows; v += blockDim.x >> f.log_team) {
    if (f.used && (__ldg(f.used + (v >> 5)) >> (v & 31) & 1)) continue;
    char* row = f.table + v * f.stride;
    const int head = static_cast<int>(min(f.bytes, static_cast<long long>(-reinterpret_cast<uintptr_t>(row) & 15)));
    const int whole = static_cast<int>((f.bytes - head) / 16);
    uint4* to = reinterpret_cast<uint4*>(row + head) + t;
#pragma unroll 4
    for (int u = t; u < whole; u += step, to += step) *to = make_uint4(0, 0, 0, 0);
    if (t) continue;
    for (int b = 0; b < f.bytes; b += f.size) {
      if (b == head) b += whole * 16;
      if (b >= f.bytes) break;
      if (f.size == 2) *reinterpret_cast<unsigned short*>(row + b) = 0;
      else *reinterpret_cast<unsigned*>(row + b) = 0;
    }
  }
}

// Ids sorted by the first cluster, SMALL_TILE ids a block in shared memory; the bitmap too.  Each pass moves a key straight into
// the block of its new place.  The other clusters' blocks write zeros.
__global__ void __launch_bounds__(SMALL_THREADS) emb_sort_small_kernel(const void* ids, int itype, int tokens, int vocab,
                                                                       long long padding, int total_bits, uint32_t* used,
                                                                       uint32_t* key_out, uint32_t* pos_out, int* status, int blocks, const EmbFill fill) {
  twa_begin(ids);
  if (static_cast<int>(blockIdx.x) >= blocks) {
    emb_fill(fill, blockIdx.x - blocks);
    return;
  }
  __shared__ unsigned long long tile[SMALL_TILE];              // key, position
  __shared__ unsigned short count[SMALL_WARPS][SMALL_BINS];
  __shared__ unsigned all_of[SMALL_BINS];                      // keys of each digit in this block
  __shared__ int warp_total[SMALL_BINS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = blockIdx.x;
  if (used) {
    for (int i = rank * SMALL_THREADS + threadIdx.x; i < (vocab + 31) / 32; i += blocks * SMALL_THREADS) used[i] = 0;
    twa_cluster_sync();
  }
  const int i0 = warp * 32 * SORT_KEYS + lane;
  unsigned long long entry[SORT_KEYS];
#pragma unroll
  for (int k = 0; k < SORT_KEYS; ++k) {
    const int t = rank * SMALL_TILE + i0 + k * 32;
    uint32_t key = 0xffffffffu;                                // beyond the tokens: after all of them
    if (t < tokens) {
      key = emb_key(ids, itype, t, vocab, padding, status);
      if (used && key < static_cast<uint32_t>(vocab)) atomicOr(&used[key >> 5], 1u << (key & 31));
    }
    entry[k] = static_cast<unsigned long long>(key) << 32 | static_cast<uint32_t>(t);
  }
  for (int shift = 32; shift < 32 + total_bits; shift += SMALL_BITS) {
    for (int d = threadIdx.x; d < SMALL_WARPS * SMALL_BINS / 2; d += SMALL_THREADS) reinterpret_cast<unsigned*>(count)[d] = 0;
    __syncthreads();
    int before_me[SORT_KEYS];                                  // equal digits of the warp's earlier keys
#pragma unroll
    for (int k = 0; k < SORT_KEYS; ++k) {
      const int d = static_cast<int>(entry[k] >> shift) & (SMALL_BINS - 1);
      const unsigned same = __match_any_sync(0xffffffffu, d);
      const int before = __popc(same & ((1u << lane) - 1));
      before_me[k] = count[warp][d] + before;
      __syncwarp();
      if (before == 0) count[warp][d] += static_cast<unsigned short>(__popc(same));
      __syncwarp();
    }
    __syncthreads();
    int here = 0;
    if (threadIdx.x < SMALL_BINS) {
      for (int w = 0; w < SMALL_WARPS; ++w) here += count[w][threadIdx.x];
      all_of[threadIdx.x] = here;
    }
    twa_cluster_sync();                                        // every block's counts are there, and its tile has been read
    // where the block's keys of each digit begin: smaller digits, then the digit in earlier blocks, then in earlier warps
    int all = 0, earlier = 0, sum = 0;
    if (threadIdx.x < SMALL_BINS) {
      for (int b = 0; b < blocks; ++b) {
        const int c = b == rank ? here : static_cast<int>(twa_remote(&all_of[threadIdx.x], b));
        if (b < rank) earlier += c;
        all += c;
      }
      sum = all;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
      }
      if (lane == 31) warp_total[warp] = sum;
    }
    __syncthreads();
    if (threadIdx.x < SMALL_BINS) {
      int at = sum - all + earlier;
      for (int w = 0; w < warp; ++w) at += warp_total[w];
      for (int w = 0; w < SMALL_WARPS; ++w) {
        const int c = count[w][threadIdx.x];
        count[w][threadIdx.x] = static_cast<unsigned short>(at);
        at += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_KEYS; ++k) {
      const int to = count[warp][static_cast<int>(entry[k] >> shift) & (SMALL_BINS - 1)] + before_me[k];
      twa_store_remote(&tile[to % SMALL_TILE], to / SMALL_TILE, entry[k]);
    }
    twa_cluster_sync();
#pragma unroll
    for (int k = 0; k < SORT_KEYS; ++k) entry[k] = tile[i0 + k * 32];
  }
#pragma unroll
  for (int k = 0; k < SORT_KEYS; ++k) {
    const int t = rank * SMALL_TILE + i0 + k * 32;
    if (t < tokens) {
      key_out[t] = static_cast<uint32_t>(entry[k] >> 32);
      pos_out[t] = static_cast<uint32_t>(entry[k]);
    }
  }
}

// One pass of the radix sort over the digit at `shift`: stable, a tile per block, and blocks that write zeros.  key_in == null: the keys are the ids'.
// Counts the next digit of every key in the tile that the key moves to (hist_next, cleared; integer sums).
__global__ void emb_scatter_kernel(const void* __restrict__ ids, int itype, int vocab, long long padding,
                                   const uint32_t* __restrict__ key_in, const uint32_t* __restrict__ pos_in, int tokens,
                                   int shift, int bits, const int* __restrict__ hist, int* __restrict__ hist_next,
                                   uint32_t* __restrict__ key_out, uint32_t* __restrict__ pos_out, int tiles,
                                   EmbFill fill) {
  twa_begin(ids, key_in, pos_in, hist, fill.used);
  if (static_cast<int>(blockIdx.x) >= tiles) {
    emb_fill(fill, blockIdx.x - tiles);
    return;
  }
  __shared__ int count[SORT_WARPS][SORT_BINS];
  __shared__ int base[SORT_BINS];
  __shared__ int warp_total[SORT_WARPS];
  const int bins = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tile = blockIdx.x;
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

// ---- sums, joins ------------------------------------------------------------------------------------
template <typename TG, int E>
__device__ __forceinline__ void emb_write(TG* to, float (&sum)[E], float scale, int accumulate) {
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] *= scale;
  if (accumulate) {
    float held[E];
    load_row<TG, E>(to, held);
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += held[e];
  }
  store_row<TG, E>(to, sum);
}

// Run `block / column_blocks` of the sorted list, columns of block % column_blocks: the rows of every id that begins in the
// run are added in order.  An id that covers some run whole leaves its sum over this run in partial[run][1] if it begins
// here, in partial[run][0] otherwise.  Blocks from sum_blocks on write zeros.
constexpr int SUM_THREADS = 128;
template <typename TD, typename TG, int E>
__global__ void __launch_bounds__(SUM_THREADS) emb_sum_kernel(const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                                              int tokens, int vocab, int dim, const TD* __restrict__ dout,
                                                              long long ldd, float scale, TG* __restrict__ dtable, long long ldg,
                                                              int accumulate, float* __restrict__ partial, int column_blocks,
                                                              int sum_blocks, EmbFill fill) {
  twa_begin(key, pos, dout, dtable, fill.used);
  if (static_cast<int>(blockIdx.x) >= sum_blocks) {
    emb_fill(fill, blockIdx.x - sum_blocks);
    return;
  }
  constexpr int P = E == 1 ? 1 : E / twa_vec<TD>;                 // packs of E elements
  constexpr int AHEAD = 8 / P;
  typedef twa_pack<TD, E == 1 ? 1 : twa_vec<TD>> Pack;
  static_assert(EMB_RUN == 32, "a lane per entry of a run");
  __shared__ uint32_t keys[2 * EMB_RUN + 1], p[2 * EMB_RUN], far;
  uint32_t* k = keys + 1;                                         // k[i]: entry first + i
  const int run = blockIdx.x / column_blocks, first = run * EMB_RUN;
  const int n = min(EMB_RUN, tokens - first), n2 = min(2 * EMB_RUN, tokens - first);
  for (int i = static_cast<int>(threadIdx.x) - 1; i < 2 * EMB_RUN; i += SUM_THREADS) {
    k[i] = first + i >= 0 && i < n2 ? key[first + i] : 0xffffffffu;
    if (i >= 0 && i < n2) p[i] = pos[first + i];
  }
  if (threadIdx.x == 0) far = first > EMB_RUN ? key[first - EMB_RUN - 1] : 0xffffffffu;    // the last entry two runs before
  __syncthreads();
  const int lane = threadIdx.x & 31;
  // the id that the run begins with, if it began before, and the one it ends with, if that goes on
  const bool before = k[-1] == k[0], after = n2 > n && k[n] == k[n - 1];
  const uint32_t lead = k[0], trail = k[n - 1];
  const bool lead_partial = before && (far == lead || (n == EMB_RUN && trail == lead));
  const bool trail_partial = after && (k[-1] == trail || (n2 == 2 * EMB_RUN && k[n2 - 1] == trail));
  const unsigned leading = __ballot_sync(0xffffffffu, lane < n && k[lane] == lead);
  const unsigned trailing = __ballot_sync(0xffffffffu, EMB_RUN + lane < n2 && k[EMB_RUN + lane] == trail);
  const int from = before && !lead_partial ? __popc(leading) : 0;
  const int to = after && !trail_partial ? n + __popc(trailing) : n;
  const int c = ((blockIdx.x - run * column_blocks) * SUM_THREADS + threadIdx.x) * E;
  if (c >= dim) return;
  float sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0f;
  for (int i0 = from; i0 < to; i0 += AHEAD) {
    Pack q[AHEAD][P];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (i0 + j < to && k[i0 + j] < static_cast<uint32_t>(vocab))
#pragma unroll
        for (int h = 0; h < P; ++h) q[j][h].load(dout + static_cast<long long>(p[i0 + j]) * ldd + c + h * (E / P));
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = i0 + j;
      if (i >= to) break;
      const uint32_t id = k[i];
      if (id >= static_cast<uint32_t>(vocab)) return;             // the rest contributes nothing
      float v[E];
#pragma unroll
      for (int h = 0; h < P; ++h) q[j][h].widen(v + h * (E / P));
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += v[e];
      const bool last = i + 1 == to;
      if (!last && k[i + 1] == id) continue;
      const bool first_part = lead_partial && id == lead;
      if (first_part || (last && trail_partial))
        store_row<float, E>(partial + (static_cast<long long>(run) * 2 + (first_part ? 0 : 1)) * dim + c, sum);
      else
        emb_write<TG, E>(dtable + static_cast<long long>(id) * ldg + c, sum, scale, accumulate);
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    }
  }
}

// The ids that begin in one of the runs JOIN_RUNS * blockIdx.x .. and cover the next run whole: their partial sums over their
// runs, JOIN_WAYS stretches of runs side by side; the columns of blockIdx.y.
constexpr int JOIN_WAYS = 8, JOIN_LANES = 32, JOIN_RUNS = 16;
template <typename TG, int E>
__global__ void __launch_bounds__(JOIN_WAYS* JOIN_LANES)
    emb_join_kernel(const uint32_t* __restrict__ key, int tokens, int vocab, int dim, float scale, TG* __restrict__ dtable,
                    long long ldg, int accumulate, const float* __restrict__ partial) {
  twa_begin(key, dtable, partial);
  __shared__ float part[JOIN_WAYS][JOIN_LANES][E + 1];
  __shared__ unsigned begins;
  const int runs = (tokens + EMB_RUN - 1) / EMB_RUN;
  if (threadIdx.x < 32) {
    const long long first = (static_cast<long long>(blockIdx.x) * JOIN_RUNS + threadIdx.x) * EMB_RUN, next = first + EMB_RUN;
    bool yes = threadIdx.x < JOIN_RUNS && next + EMB_RUN <= tokens;
    if (yes) {
      const uint32_t id = key[next - 1], end = key[next + EMB_RUN - 1], before = first > 0 ? key[first - 1] : 0xffffffffu;
      yes = id < static_cast<uint32_t>(vocab) && end == id && before != id;
    }
    const unsigned all = __ballot_sync(0xffffffffu, yes);
    if (threadIdx.x == 0) begins = all;
  }
  __syncthreads();
  const int lane = threadIdx.x % JOIN_LANES, way = threadIdx.x / JOIN_LANES;
  for (unsigned left = begins; left; left &= left - 1) {
    const int from = blockIdx.x * JOIN_RUNS + __ffs(left) - 1;
    const uint32_t id = key[from * static_cast<long long>(EMB_RUN) + EMB_RUN - 1];
    // its runs are from .. to - 1: all threads probe the runs after `low`, ever closer together
    int low = from + 1, high = runs;
    while (low + 1 < high) {
      const int step = (high - low - 1 + JOIN_WAYS * JOIN_LANES - 1) / (JOIN_WAYS * JOIN_LANES);
      const long long probe = low + (threadIdx.x + 1LL) * step;
      const int inside = __syncthreads_count(probe < high && key[probe * EMB_RUN] == id);
      const long long beyond = low + (inside + 1LL) * step;
      low += inside * step;
      if (beyond < high) high = static_cast<int>(beyond);
    }
    const int to = low + 1;
    const int each = (to - from + JOIN_WAYS - 1) / JOIN_WAYS;
    const int a = from + way * each, b = min(to, a + each);
    const int c = (blockIdx.y * JOIN_LANES + lane) * E;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    if (c < dim)
      for (int r = a; r < b; ++r) {
        float v[E];
        load_row<float, E>(partial + (static_cast<long long>(r) * 2 + (r == from ? 1 : 0)) * dim + c, v);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += v[e];
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
  const int parts = static_cast<int>(twa_ceil_div(dim, packs ? 8 * 32 * FWD_UNITS<8> : 32 * FWD_UNITS<1>));
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(tokens * parts, FWD_WARPS));
  if (packs)
    twa_launch(ctx->stream, embedding_kernel<TT, TO, 8>, blocks, 32 * FWD_WARPS, 0, static_cast<const TT*>(table), ldt, vocab, ids, itype,
                                                                          tokens, dim, scale, static_cast<TO*>(out), ldo, parts,
                                                                          ctx->d_status);
  else
    twa_launch(ctx->stream, embedding_kernel<TT, TO, 1>, blocks, 32 * FWD_WARPS, 0, static_cast<const TT*>(table), ldt, vocab, ids, itype,
                                                                          tokens, dim, scale, static_cast<TO*>(out), ldo, parts,
                                                                          ctx->d_status);
}

// Zeros written beside the one launch that sorts in shared memory: 160 MB, or 128 where rows do not begin and end on 16 bytes, which are
// written more slowly.  A single block (up to 2048 ids) sorts in half the time of a cluster: at most half of the table then (but
// 48 MB), because the sums that follow hide the rest if they take a run of ids and more.  In us, bfloat16 rows into
// float32 or bfloat16 (b) tables, by MB beside the sort:
//                         64    96   128   160                              32    64    96   128   160
//   16384, 50272 x 2048   86.9  84.8  83.3  81.6      2048, 50272 x 2048     73.2  70.5  66.6  66.8  67.7
//   16384, 128000 x 777   95.4  92.2  92.8  94.4      2048, 128000 x 777     76.6  71.8  72.4  73.9  75.1
//   16384, 128000 x 1024b 69.9  66.0  63.1  62.9      2048, 128000 x 1024b   62.0  56.8  54.9  54.3  53.6
//    4096, 128000 x 777   78.2  75.1  74.4  75.5      2048, 120000 x 256     37.0  34.8  37.4  39.8  39.8
//    4096, 32000 x 4096   94.6  93.2  92.3  91.7        64, 120000 x 256     28.5  27.2  30.9  34.0  34.0
// and half / all of the table: 1, 50272 x 768b 20.9 / 19.5; 64, 32003 x 129b 21.1 / 18.8; 2048, 24000 x 1024b 29.0 / 27.7.
long long emb_beside(const EmbFill& fill, int tokens, int blocks) {
  const bool whole = ((reinterpret_cast<uintptr_t>(fill.table) | fill.stride | fill.bytes) & 15) == 0;
  const long long half = fill.bytes * fill.row1 / 2, least = 48LL << 20, most = (whole ? 160LL : 128LL) << 20;
  if (blocks > 1 || tokens < EMB_RUN || half > most) return most;
  return half > least ? half : least;
}

// The number of blocks that write the zeros of rows row0 .. of `fill` within `budget` bytes (0: all that are left); the
// rows are taken off `left`.
unsigned emb_fill_blocks(const EmbFill& left, long long budget, EmbFill* part) {
  *part = left;
  if (budget) {
    const long long rows = budget / left.bytes / left.each * left.each;
    if (left.row0 + rows < left.row1) part->row1 = static_cast<int>(left.row0 + rows);
  }
  return static_cast<unsigned>(twa_ceil_div(part->row1 - part->row0, left.each));
}

template <typename TD, typename TG, int E>
void launch_sums(twa_ctx* ctx, const EmbSpace& s, const uint32_t* key, const uint32_t* pos, int tokens, int vocab, int dim,
                 const void* dout, int64_t ldd, float scale, void* dtable, int64_t ldg, int accumulate, const EmbFill& fill) {
  TG* g = static_cast<TG*>(dtable);
  const unsigned runs = static_cast<unsigned>(twa_ceil_div(tokens, EMB_RUN));
  const unsigned column_blocks = static_cast<unsigned>(twa_ceil_div(dim, E * SUM_THREADS));
  EmbFill rest;
  const unsigned zeros = emb_fill_blocks(fill, 0, &rest);
  if (runs * column_blocks + zeros)
    twa_launch(ctx->stream, emb_sum_kernel<TD, TG, E>, runs * column_blocks + zeros, SUM_THREADS, 0, key, pos, tokens, vocab, dim, static_cast<const TD*>(dout), ldd, scale, g, ldg, accumulate, s.partial, column_blocks,
        runs * column_blocks, rest);
  if (tokens >= 2 * EMB_RUN)
    twa_launch(ctx->stream, emb_join_kernel<TG, E>, dim3(static_cast<unsigned>(twa_ceil_div(runs - 1, JOIN_RUNS)), static_cast<unsigned>(twa_ceil_div(dim, E * JOIN_LANES))), JOIN_WAYS * JOIN_LANES, 0, key, tokens, vocab, dim, scale, g, ldg, accumulate, s.partial);
}

template <typename TD, typename TG>
void launch_sums_any(twa_ctx* ctx, bool packs, const EmbSpace& s, const uint32_t* key, const uint32_t* pos, int tokens, int vocab,
                     int dim, const void* dout, int64_t ldd, float scale, void* dtable, int64_t ldg, int accumulate,
                     const EmbFill& fill) {
  if (packs) launch_sums<TD, TG, 8>(ctx, s, key, pos, tokens, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate, fill);
  else launch_sums<TD, TG, 1>(ctx, s, key, pos, tokens, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate, fill);
}

}  // namespace

extern "C" {

int twa_embedding(twa_ctx* ctx, const void* table, int64_t ldt, twa_dtype t_dtype, int vocab, int dim, const void* ids,
                  twa_itype id_type, int64_t tokens, float scale, void* out, int64_t ldo, twa_dtype out_dtype) {
  if (!ctx || !twa_dtype_ok(t_dtype) || !twa_dtype_ok(out_dtype) || !twa_itype_ok(id_type)) return TWA_ERR_INVALID_ARG;
  if (vocab < 1 || dim < 1 || tokens < 0) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_EMBEDDING_MAX_TOKENS || dim > TWA_EMBEDDING_MAX_DIM || vocab > TWA_EMBEDDING_MAX_VOCAB) return TWA_ERR_UNSUPPORTED;
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
  if (tokens < 0 || tokens > TWA_EMBEDDING_MAX_TOKENS || vocab < 1 || vocab > TWA_EMBEDDING_MAX_VOCAB || dim < 1 || dim > TWA_EMBEDDING_MAX_DIM) return 0;
  return emb_space(nullptr, tokens, vocab, dim).bytes;
}

int twa_embedding_backward(twa_ctx* ctx, const void* dout, int64_t ldd, twa_dtype d_dtype, const void* ids, twa_itype id_type,
                           int64_t tokens, int vocab, int dim, float scale, int64_t padding_id, void* dtable, int64_t ldg,
                           twa_dtype g_dtype, int accumulate, void* ws, size_t ws_bytes) {
  if (!ctx || !twa_dtype_ok(d_dtype) || !twa_dtype_ok(g_dtype) || !twa_itype_ok(id_type)) return TWA_ERR_INVALID_ARG;
  if (vocab < 1 || dim < 1 || tokens < 0 || accumulate < 0 || accumulate > 1) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_EMBEDDING_MAX_TOKENS || dim > TWA_EMBEDDING_MAX_DIM || vocab > TWA_EMBEDDING_MAX_VOCAB) return TWA_ERR_UNSUPPORTED;
  if (!dtable || ldg < dim || (tokens && (!dout || !ids || ldd < dim))) return TWA_ERR_INVALID_ARG;
  const size_t ds = twa_dtype_size(d_dtype), gs = twa_dtype_size(g_dtype);
  if (twa_misaligned_to(dtable, gs) || (tokens && (twa_misaligned_to(dout, ds) || twa_misaligned_to(ids, twa_itype_size(id_type)))))
    return TWA_ERR_MISALIGNED;
  if (!ws || ws_bytes < twa_embedding_workspace_bytes(tokens, vocab, dim)) return TWA_ERR_WORKSPACE;
  if (twa_misaligned_to(ws, 16)) return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  const EmbSpace s = emb_space(ws, tokens, vocab, dim);
  const int n = static_cast<int>(tokens), tiles = static_cast<int>(twa_ceil_div(tokens, SORT_TILE));
  const bool packs = dim % 8 == 0 && emb_packs(dout, ldd, ds) && emb_packs(dtable, ldg, gs);
  int total_bits = 1;
  while (total_bits < 32 && (static_cast<long long>(vocab) >> total_bits)) ++total_bits;      // keys 0 .. vocab
  EmbFill fill = {static_cast<char*>(dtable), static_cast<long long>(ldg * gs), static_cast<long long>(dim * gs), s.used, 0,
                  accumulate ? 0 : vocab, 1, static_cast<int>(gs), 0};
  while (fill.log_team < FILL_TEAM && 16LL << fill.log_team < fill.bytes) ++fill.log_team;
  if (fill.bytes < FILL_BYTES) fill.each = static_cast<int>(FILL_BYTES / fill.bytes);
  int at = 0;
  if (n <= SMALL_TOKENS && vocab <= SMALL_VOCAB) {
    const int blocks = n <= SMALL_TILE ? 1 : (n <= 2 * SMALL_TILE ? 2 : (n <= 4 * SMALL_TILE ? 4 : 8));
    EmbFill part;
    const unsigned zeros = emb_fill_blocks(fill, emb_beside(fill, n, blocks), &part);
    part.used = nullptr;
    const unsigned grid = blocks + static_cast<unsigned>(twa_ceil_div(zeros, blocks)) * blocks;
    const cudaError_t launched =
        twa_launch_clusters(ctx->stream, emb_sort_small_kernel, grid, blocks, SMALL_THREADS, 0, ids, id_type, n, vocab, padding_id,
                            total_bits, accumulate ? nullptr : s.used, s.key[at], s.pos[at], ctx->d_status, blocks, part);
    TWA_CUDA_OK(ctx, launched);
    fill.row0 = part.row1;
  } else {
    TWA_CUDA_OK(ctx, cudaMemsetAsync(s.used, 0, reinterpret_cast<char*>(s.key[0]) - reinterpret_cast<char*>(s.used), ctx->stream));
    const int passes = (total_bits + SORT_MAX_BITS - 1) / SORT_MAX_BITS, bits = (total_bits + passes - 1) / passes;
    if (n)
      twa_launch(ctx->stream, emb_count_kernel, tiles, SORT_THREADS, 0, ids, id_type, n, vocab, padding_id, bits, s.used, s.hist[0],
                                                                ctx->d_status);
    for (int p = 0; n && p < passes; ++p) {
      int* next = p + 1 < passes ? s.hist[(p + 1) & 1] : nullptr;
      if (p >= 1 && next) TWA_CUDA_OK(ctx, cudaMemsetAsync(next, 0, sizeof(int) * SORT_BINS * tiles, ctx->stream));
      EmbFill part;
      const unsigned zeros = emb_fill_blocks(fill, FILL_BESIDE_SORT, &part);
      twa_launch(ctx->stream, emb_scatter_kernel, tiles + zeros, SORT_THREADS, 0, ids, id_type, vocab, padding_id, p ? s.key[at] : nullptr,
                                                                          p ? s.pos[at] : nullptr, n, p * bits, bits,
                                                                          s.hist[p & 1], next, s.key[at ^ 1], s.pos[at ^ 1], tiles,
                                                                          part);
      fill.row0 = part.row1;
      at ^= 1;
    }
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  const bool db = d_dtype == TWA_BF16, gb = g_dtype == TWA_BF16;
  const uint32_t *key = s.key[at], *pos = s.pos[at];
  if (db && gb) launch_sums_any<bf16, bf16>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate, fill);
  else if (db) launch_sums_any<bf16, float>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate, fill);
  else if (gb) launch_sums_any<float, bf16>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate, fill);
  else launch_sums_any<float, float>(ctx, packs, s, key, pos, n, vocab, dim, dout, ldd, scale, dtable, ldg, accumulate, fill);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
