// Gated linear recurrence, both directions; the forms that are used here stand in twa_scan.cuh.
//
//   forward    h_t = a_t h_{t-1} + (1 - a_t) x_t,   a_t = sigmoid(f_t)
//   backward   G_t = dh_t + a_{t+1} G_{t+1},   dx_t = (1 - a_t) G_t,   df_t = a_t (1 - a_t) (h_{t-1} - x_t) G_t
//
// Backward the states before every row are taken again from those that the forward pass kept in float32, one every 64 rows, and
// what goes from row to row is k_t = a_t G_t, affine in the one that enters: k = A k_in + M with the same A as forward.
#include "twa_scan.cuh"

namespace {

// Maps of the segments of a tile, and of the tiles of a cluster's blocks: twice, so that the next ones go beside those being read.
template <int MAPS>
struct Joins {
  twa_f2 seg[2][SCAN_WARPS][MAPS][32], tile[2][MAX_CLUSTER][MAPS][32];
};

// Where a thread stands: its lane's channels c and c + 1, of which n exist, and its block's rank along the sequence.
struct Place {
  int lane, warp, c, n, rank, ranks;
  __device__ __forceinline__ Place(const ScanArgs& a, int slice) {
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    c = slice * SCAN_CHANNELS + 2 * lane;
    const int left = a.channels - c;
    n = left < 0 ? 0 : (left < 2 ? left : 2);
    ranks = a.cluster;
    rank = ranks > 1 ? static_cast<int>(twa_cluster_rank()) : 0;
  }
};

// The blocks of a cluster tell each other what their tiles make of a state: every block's warp 0 joins its segments' maps and
// stores the tile's into every block.  FORWARD: segments in their order, otherwise from the last.  A map is (A, B): v -> A v + B; the
// B is the last of the MAPS that a segment leaves.
template <bool FORWARD, int MAPS>
__device__ __forceinline__ void share_tile(Joins<MAPS>& joins, const Place& at, int turn) {
  if (at.warp == 0) {
    twa_f2 A = twa_pair(1.0f), B = 0;
#pragma unroll
    for (int i = 0; i < SCAN_WARPS; ++i) {
      const int w = FORWARD ? i : SCAN_WARPS - 1 - i;
      const twa_f2 m = joins.seg[turn][w][0][at.lane];
      A = twa_mul2(m, A);
      B = twa_fma2(m, B, joins.seg[turn][w][MAPS - 1][at.lane]);
    }
    for (int r = 0; r < at.ranks; ++r) {
      twa_store_remote(&joins.tile[turn][at.rank][0][at.lane], r, A);
      twa_store_remote(&joins.tile[turn][at.rank][1][at.lane], r, B);
    }
  }
  twa_cluster_sync();
}

template <typename T, int FEED>
struct ScanForward {
  static constexpr int MAPS = 2, STAGES = FEED == BY_ELEMENTS ? 1 : (sizeof(T) == 2 ? 4 : 3);
  static constexpr bool PACKED = FEED != BY_ELEMENTS;
  typedef Ring<T, FEED, 2, STAGES> Rows;
  const ScanArgs& a;
  const Place at;
  twa_f2 A[SEG], L[SEG];                           // of the rows up to each

  __device__ __forceinline__ ScanForward(const ScanArgs& args, int slice) : a(args), at(args, slice) {}

  __device__ __forceinline__ void row(int i, const Pair<T>& x, const Pair<T>& f, twa_f2& s, twa_f2& l) {
    const twa_f2 n = scan_gate<T>(f);
    s = scan_decay(n, s);
    l = scan_step(n, l, x.both());
    A[i] = s;
    L[i] = l;
  }
  __device__ __forceinline__ void store(long long first, int rows, twa_f2 in) {
    T* h = static_cast<T*>(a.h) + first * a.ldh + at.c;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows && at.n > 0) {
        float lo, hi;
        twa_unpair(twa_fma2(A[i], in, L[i]), lo, hi);
        Pair<T>::template store<PACKED>(h + i * a.ldh, lo, hi, at.n);
      }
  }

  // A sequence of at most SEG rows, by one warp.
  __device__ __forceinline__ void brief(const Span& s, int seq) {
    const int rows = static_cast<int>(s.len);
    const T* x = static_cast<const T*>(a.x) + s.begin * a.ldx + at.c;
    const T* f = static_cast<const T*>(a.f) + s.begin * a.ldf + at.c;
    Pair<T> rx[SEG], rf[SEG];
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows && at.n > 0) {
        rx[i].template load<PACKED>(x + i * a.ldx, at.n);
        rf[i].template load<PACKED>(f + i * a.ldf, at.n);
      }
    const twa_f2 in = scan_state(a.h0, seq, a.channels, at.c, at.n);
    if (rows) scan_keep(a.states, scan_slot(s, seq), a.channels, at.c, at.n, in);
    twa_f2 A1 = twa_pair(1.0f), L1 = 0;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows) row(i, rx[i], rf[i], A1, L1);
    store(s.begin, rows, in);
    scan_keep(a.h_last, seq, a.channels, at.c, at.n, twa_fma2(A1, in, L1));
  }

  // A sequence by the whole cluster.
  __device__ __forceinline__ void whole(const Span& s, int seq, char* shared, Joins<MAPS>& joins, int& turn) {
    Rows ring(shared, at.warp);
    const long long stride = static_cast<long long>(SCAN_ROWS) * at.ranks;
    const int left = a.channels - (at.c - 2 * at.lane);                   // channels from this slice's first on
    long long ahead = at.rank * SCAN_ROWS + at.warp * SEG;                // row of the next segment to be fetched
    auto rows_at = [&](long long r) { return static_cast<int>(s.len - r < SEG ? (s.len - r < 0 ? 0 : s.len - r) : SEG); };
    auto fetch = [&]() {
      const int rows = rows_at(ahead);
      if (rows) {
        ring.copy(0, static_cast<const T*>(a.x) + (s.begin + ahead) * a.ldx + (at.c - 2 * at.lane), a.ldx, rows, left);
        ring.copy(1, static_cast<const T*>(a.f) + (s.begin + ahead) * a.ldf + (at.c - 2 * at.lane), a.ldf, rows, left);
      }
      ring.filled();
      ahead += stride;
    };
#pragma unroll
    for (int i = 0; i < Rows::AHEAD; ++i) fetch();
    twa_f2 state = scan_state(a.h0, seq, a.channels, at.c, at.n);
    long long slot = scan_slot(s, seq) + at.rank;
    for (long long t = at.rank * SCAN_ROWS; t - at.rank * SCAN_ROWS < s.len; t += stride, slot += at.ranks) {
      const long long mine = t + at.warp * SEG;
      const int rows = rows_at(mine);
      ring.wait();
      fetch();
      twa_f2 A1 = twa_pair(1.0f), L1 = 0;
      if (rows == SEG) {
#pragma unroll
        for (int i = 0; i < SEG; ++i) row(i, ring.get(0, i), ring.get(1, i), A1, L1);
      } else {
#pragma unroll
        for (int i = 0; i < SEG; ++i)
          if (i < rows) row(i, ring.get(0, i), ring.get(1, i), A1, L1);
      }
      ring.done();
      joins.seg[turn][at.warp][0][at.lane] = A1;
      joins.seg[turn][at.warp][1][at.lane] = L1;
      __syncthreads();
      twa_f2 in = state;
      if (at.ranks > 1) {
        share_tile<true>(joins, at, turn);
        for (int r = 0; r < at.ranks; ++r) {
          if (r == at.rank) in = state;
          state = twa_fma2(joins.tile[turn][r][0][at.lane], state, joins.tile[turn][r][1][at.lane]);
        }
        if (at.warp == 0 && t < s.len) scan_keep(a.states, slot, a.channels, at.c, at.n, in);
        for (int w = 0; w < at.warp; ++w) in = twa_fma2(joins.seg[turn][w][0][at.lane], in, joins.seg[turn][w][1][at.lane]);
      } else {
        if (at.warp == 0) scan_keep(a.states, slot, a.channels, at.c, at.n, state);
#pragma unroll
        for (int w = 0; w < SCAN_WARPS; ++w) {
          if (w == at.warp) in = state;
          state = twa_fma2(joins.seg[turn][w][0][at.lane], state, joins.seg[turn][w][1][at.lane]);
        }
      }
      turn ^= 1;
      store(s.begin + mine, rows, in);
    }
    if (at.warp == 0 && at.rank == 0) scan_keep(a.h_last, seq, a.channels, at.c, at.n, state);
  }
};

template <typename T, int FEED>
struct ScanBackward {
  static constexpr int MAPS = 3, STAGES = FEED == BY_ELEMENTS ? 1 : (sizeof(T) == 2 ? 3 : 2);      // maps: A, L, M
  static constexpr bool PACKED = FEED != BY_ELEMENTS;
  typedef Ring<T, FEED, 3, STAGES> Rows;
  const ScanArgs& a;
  const Place at;
  twa_f2 n[SEG], d[SEG];                           // gates; h_{t-1} - x_t

  __device__ __forceinline__ ScanBackward(const ScanArgs& args, int slice) : a(args), at(args, slice) {}

  // Gradients of a row from g = dh + k, where k is what comes from the rows behind it; k becomes this row's.
  __device__ __forceinline__ void back(int i, T* dx, T* df, twa_f2 dh, twa_f2& k) {
    const twa_f2 g = twa_add2(dh, k);
    float g0, g1, n0, n1, d0, d1;
    twa_unpair(g, g0, g1);
    twa_unpair(n[i], n0, n1);
    twa_unpair(d[i], d0, d1);
    k = scan_decay(n[i], g);
    if (at.n > 0) {
      Pair<T>::template store<PACKED>(dx + i * a.lddx, fmaf(-n0, g0, scan_open(n0) ? 0.0f : g0), fmaf(-n1, g1, scan_open(n1) ? 0.0f : g1), at.n);
      const float s0 = fabsf(n0), s1 = fabsf(n1);
      Pair<T>::template store<PACKED>(df + i * a.lddf, fmaf(-s0, s0, s0) * d0 * g0, fmaf(-s1, s1, s1) * d1 * g1, at.n);
    }
  }

  __device__ __forceinline__ void brief(const Span& s, int seq) {
    const int rows = static_cast<int>(s.len);
    const T* x = static_cast<const T*>(a.x) + s.begin * a.ldx + at.c;
    const T* f = static_cast<const T*>(a.f) + s.begin * a.ldf + at.c;
    const T* g = static_cast<const T*>(a.dh) + s.begin * a.lddh + at.c;
    Pair<T> rx[SEG], rf[SEG], rd[SEG];
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows && at.n > 0) {
        rx[i].template load<PACKED>(x + i * a.ldx, at.n);
        rf[i].template load<PACKED>(f + i * a.ldf, at.n);
        rd[i].template load<PACKED>(g + i * a.lddh, at.n);
      }
    twa_f2 h = rows ? scan_state(a.states, scan_slot(s, seq), a.channels, at.c, at.n) : 0;
    twa_f2 k = scan_state(a.d_last, seq, a.channels, at.c, at.n);
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows) {
        n[i] = scan_gate<T>(rf[i]);
        d[i] = scan_minus(h, rx[i].both());
        h = scan_step(n[i], h, rx[i].both());
      }
    T* dx = static_cast<T*>(a.dx) + s.begin * a.lddx + at.c;
    T* df = static_cast<T*>(a.df) + s.begin * a.lddf + at.c;
#pragma unroll
    for (int i = SEG - 1; i >= 0; --i)
      if (i < rows) back(i, dx, df, rd[i].both(), k);
    scan_keep(a.dh0, seq, a.channels, at.c, at.n, k);
  }

  __device__ __forceinline__ void whole(const Span& s, int seq, char* shared, Joins<MAPS>& joins, int& turn) {
    Rows ring(shared, at.warp);
    const long long stride = static_cast<long long>(SCAN_ROWS) * at.ranks;
    const long long rounds = (s.len + stride - 1) / stride;
    const int left = a.channels - (at.c - 2 * at.lane);
    long long ahead = (rounds - 1) * stride + at.rank * SCAN_ROWS + at.warp * SEG;
    auto rows_at = [&](long long r) { return static_cast<int>(s.len - r < SEG ? (s.len - r < 0 ? 0 : s.len - r) : SEG); };
    auto fetch = [&]() {
      const int rows = ahead < 0 ? 0 : rows_at(ahead);
      if (rows) {
        ring.copy(0, static_cast<const T*>(a.x) + (s.begin + ahead) * a.ldx + (at.c - 2 * at.lane), a.ldx, rows, left);
        ring.copy(1, static_cast<const T*>(a.f) + (s.begin + ahead) * a.ldf + (at.c - 2 * at.lane), a.ldf, rows, left);
        ring.copy(2, static_cast<const T*>(a.dh) + (s.begin + ahead) * a.lddh + (at.c - 2 * at.lane), a.lddh, rows, left);
      }
      ring.filled();
      ahead -= stride;
    };
#pragma unroll
    for (int i = 0; i < Rows::AHEAD; ++i) fetch();
    twa_f2 k = scan_state(a.d_last, seq, a.channels, at.c, at.n);
    for (long long round = rounds - 1; round >= 0; --round) {
      const long long t = round * stride + at.rank * SCAN_ROWS, mine = t + at.warp * SEG;
      const int rows = rows_at(mine);
      twa_f2 h = t < s.len ? scan_state(a.states, scan_slot(s, seq) + round * at.ranks + at.rank, a.channels, at.c, at.n) : 0;
      ring.wait();
      fetch();
      twa_f2 A1 = twa_pair(1.0f), L1 = 0, M1 = 0;
#pragma unroll
      for (int i = 0; i < SEG; ++i)
        if (i < rows) {
          n[i] = scan_gate<T>(ring.get(1, i));
          A1 = scan_decay(n[i], A1);
          L1 = scan_step(n[i], L1, ring.get(0, i).both());
        }
#pragma unroll
      for (int i = SEG - 1; i >= 0; --i)
        if (i < rows) M1 = scan_decay(n[i], twa_add2(ring.get(2, i).both(), M1));
      joins.seg[turn][at.warp][0][at.lane] = A1;
      joins.seg[turn][at.warp][1][at.lane] = L1;
      joins.seg[turn][at.warp][2][at.lane] = M1;
      __syncthreads();
      twa_f2 in = k;
      if (at.ranks > 1) {
        share_tile<false>(joins, at, turn);
        for (int r = at.ranks - 1; r >= 0; --r) {
          if (r == at.rank) in = k;
          k = twa_fma2(joins.tile[turn][r][0][at.lane], k, joins.tile[turn][r][1][at.lane]);
        }
        for (int w = SCAN_WARPS - 1; w > at.warp; --w) in = twa_fma2(joins.seg[turn][w][0][at.lane], in, joins.seg[turn][w][2][at.lane]);
      } else {
#pragma unroll
        for (int w = SCAN_WARPS - 1; w >= 0; --w) {
          if (w == at.warp) in = k;
          k = twa_fma2(joins.seg[turn][w][0][at.lane], k, joins.seg[turn][w][2][at.lane]);
        }
      }
      for (int w = 0; w < at.warp; ++w) h = twa_fma2(joins.seg[turn][w][0][at.lane], h, joins.seg[turn][w][1][at.lane]);
      turn ^= 1;
      T* dx = static_cast<T*>(a.dx) + (s.begin + mine) * a.lddx + at.c;
      T* df = static_cast<T*>(a.df) + (s.begin + mine) * a.lddf + at.c;
#pragma unroll
      for (int i = 0; i < SEG; ++i)
        if (i < rows) {
          const twa_f2 x = ring.get(0, i).both();
          d[i] = scan_minus(h, x);
          h = scan_step(n[i], h, x);
        }
#pragma unroll
      for (int i = SEG - 1; i >= 0; --i)
        if (i < rows) back(i, dx, df, ring.get(2, i).both(), in);
      ring.done();
    }
    if (at.warp == 0 && at.rank == 0) scan_keep(a.dh0, seq, a.channels, at.c, at.n, k);
  }
};

// GROUP sequences of a slice of channels a block.  The ones of at most SEG rows go to one warp each, the others to the block.
template <typename Direction, int GROUP>
__device__ __forceinline__ void scan_block(const ScanArgs& a) {
  extern __shared__ __align__(16) char shared[];
  __shared__ Joins<Direction::MAPS> joins;
  const unsigned task = blockIdx.x / a.cluster;
  const int slice = task % a.slices, first = task / a.slices * GROUP;
  Direction d(a, slice);
  if (a.cluster > 1) twa_cluster_sync();           // no block stores into one that has not begun
  if (GROUP > 1) {
    const int seq = first + d.at.warp;
    if (seq < a.sequences) {
      const Span s = scan_span(a, seq, slice == 0 && d.at.lane == 0);
      if (s.len >= 0 && s.len <= SEG) d.brief(s, seq);
    }
  }
  int turn = 0;
  for (int g = 0; g < GROUP; ++g) {
    const int seq = first + g;
    if (seq >= a.sequences) break;
    const Span s = scan_span(a, seq, GROUP == 1 && slice == 0 && threadIdx.x == 0);
    if (s.len > SEG || (GROUP == 1 && s.len >= 0)) d.whole(s, seq, shared, joins, turn);
  }
}

template <typename T, int FEED, int GROUP>
__global__ void __launch_bounds__(SCAN_THREADS, 2) scan_forward_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.starts, a.h0);
  scan_block<ScanForward<T, FEED>, GROUP>(a);
}
template <typename T, int FEED, int GROUP>
__global__ void __launch_bounds__(SCAN_THREADS, 2) scan_backward_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.dh, a.starts, a.states, a.d_last);
  scan_block<ScanBackward<T, FEED>, GROUP>(a);
}

// How rows of two pointers and strides can be fetched together.
int scan_feed(const void* p, long long ld, size_t size, int channels, int so_far) {
  if (so_far == BY_UNITS && (channels * size % 16 || twa_misaligned_to(p, 16) || ld * size % 16)) so_far = BY_PAIRS;
  if (so_far == BY_PAIRS && (channels % 2 || twa_misaligned_to(p, 2 * size) || ld % 2)) so_far = BY_ELEMENTS;
  return so_far;
}
// Stores go by pairs at most.
int scan_feed_out(const void* p, long long ld, size_t size, int so_far) {
  return so_far != BY_ELEMENTS && (twa_misaligned_to(p, 2 * size) || ld % 2) ? BY_ELEMENTS : so_far;
}

template <typename T, int FEED, int GROUP>
cudaError_t scan_launch(twa_ctx* ctx, const ScanArgs& a, bool back) {
  auto kernel = back ? scan_backward_kernel<T, FEED, GROUP> : scan_forward_kernel<T, FEED, GROUP>;
  const size_t smem = back ? ScanBackward<T, FEED>::Rows::BLOCK_BYTES : ScanForward<T, FEED>::Rows::BLOCK_BYTES;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.sequences, GROUP) * a.slices * a.cluster);
  return twa_launch_clusters(ctx->stream, kernel, blocks, a.cluster, SCAN_THREADS, smem, a);
}
template <typename T>
cudaError_t scan_launch(twa_ctx* ctx, ScanArgs& a, bool back, int feed) {
  const bool brief = a.tokens <= 2LL * SEG * a.sequences;
  a.cluster = 1;
  while (!brief && a.cluster < MAX_CLUSTER && a.tokens > 2LL * a.cluster * SCAN_ROWS * a.sequences &&
         static_cast<long long>(a.sequences) * a.slices * a.cluster < ctx->sm_count)
    a.cluster *= 2;
  if (brief)
    return feed == BY_UNITS ? scan_launch<T, BY_UNITS, SHORT_GROUP>(ctx, a, back)
                            : (feed == BY_PAIRS ? scan_launch<T, BY_PAIRS, SHORT_GROUP>(ctx, a, back) : scan_launch<T, BY_ELEMENTS, SHORT_GROUP>(ctx, a, back));
  return feed == BY_UNITS ? scan_launch<T, BY_UNITS, 1>(ctx, a, back)
                          : (feed == BY_PAIRS ? scan_launch<T, BY_PAIRS, 1>(ctx, a, back) : scan_launch<T, BY_ELEMENTS, 1>(ctx, a, back));
}

// Arguments that both directions have.
int scan_check(twa_ctx* ctx, int dtype, int64_t tokens, int channels, const void* starts, int s_type, int sequences) {
  if (!ctx || !twa_dtype_ok(dtype) || tokens < 0 || channels < 1 || sequences < 0 || (starts && !twa_itype_ok(s_type))) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_SCAN_MAX_TOKENS || channels > TWA_SCAN_MAX_CHANNELS || sequences > TWA_SCAN_MAX_SEQUENCES) return TWA_ERR_UNSUPPORTED;
  if (!starts && (sequences ? tokens % sequences : tokens)) return TWA_ERR_INVALID_ARG;
  if (starts && twa_misaligned_to(starts, twa_itype_size(s_type))) return TWA_ERR_MISALIGNED;
  // blocks of a launch
  if (static_cast<long long>(sequences) * twa_ceil_div(channels, SCAN_CHANNELS) * MAX_CLUSTER > 0x7FFFFFFFLL) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

}  // namespace

extern "C" {

size_t twa_gated_scan_states_bytes(int64_t tokens, int sequences, int channels) {
  if (tokens < 0 || tokens > TWA_SCAN_MAX_TOKENS || sequences < 0 || sequences > TWA_SCAN_MAX_SEQUENCES || channels < 1 ||
      channels > TWA_SCAN_MAX_CHANNELS)
    return 0;
  return static_cast<size_t>(tokens / SCAN_ROWS + sequences) * channels * sizeof(float);
}

int twa_gated_scan(twa_ctx* ctx, const void* x, int64_t ldx, const void* f, int64_t ldf, twa_dtype dtype, int64_t tokens, int channels,
                   const void* starts, twa_itype s_type, int sequences, const float* h0, void* h, int64_t ldh, float* h_last, void* states,
                   size_t states_bytes) {
  const int rc = scan_check(ctx, dtype, tokens, channels, starts, s_type, sequences);
  if (rc) return rc;
  if (sequences == 0) return TWA_OK;
  if (tokens && (!x || !f || !h || ldx < channels || ldf < channels || ldh < channels)) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(h0, 4) || twa_misaligned_to(h_last, 4) ||
      (tokens && (twa_misaligned_to(x, size) || twa_misaligned_to(f, size) || twa_misaligned_to(h, size))))
    return TWA_ERR_MISALIGNED;
  if (states && states_bytes < twa_gated_scan_states_bytes(tokens, sequences, channels)) return TWA_ERR_WORKSPACE;
  if (twa_misaligned_to(states, 16)) return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  ScanArgs a = {};
  a.x = x, a.ldx = ldx, a.f = f, a.ldf = ldf, a.h = h, a.ldh = ldh;
  a.tokens = tokens, a.channels = channels, a.starts = starts, a.s_type = s_type, a.sequences = sequences;
  a.slices = static_cast<int>(twa_ceil_div(channels, SCAN_CHANNELS));
  a.h0 = h0, a.h_last = h_last, a.states = static_cast<float*>(states), a.status = ctx->d_status;
  const int feed = scan_feed_out(h, ldh, size, scan_feed(f, ldf, size, channels, scan_feed(x, ldx, size, channels, BY_UNITS)));
  TWA_CUDA_OK(ctx, dtype == TWA_BF16 ? scan_launch<bf16>(ctx, a, false, feed) : scan_launch<float>(ctx, a, false, feed));
  return TWA_OK;
}

int twa_gated_scan_backward(twa_ctx* ctx, const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* f, int64_t ldf, twa_dtype dtype,
                            int64_t tokens, int channels, const void* starts, twa_itype s_type, int sequences, const void* states,
                            size_t states_bytes, const float* d_last, void* dx, int64_t lddx, void* df, int64_t lddf, float* dh0) {
  const int rc = scan_check(ctx, dtype, tokens, channels, starts, s_type, sequences);
  if (rc) return rc;
  if (sequences == 0) return TWA_OK;
  if (tokens && (!dh || !x || !f || !dx || !df || lddh < channels || ldx < channels || ldf < channels || lddx < channels || lddf < channels))
    return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(d_last, 4) || twa_misaligned_to(dh0, 4) ||
      (tokens && (twa_misaligned_to(dh, size) || twa_misaligned_to(x, size) || twa_misaligned_to(f, size) || twa_misaligned_to(dx, size) ||
                  twa_misaligned_to(df, size))))
    return TWA_ERR_MISALIGNED;
  if (!states || states_bytes < twa_gated_scan_states_bytes(tokens, sequences, channels)) return TWA_ERR_WORKSPACE;
  if (twa_misaligned_to(states, 16)) return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  ScanArgs a = {};
  a.dh = dh, a.lddh = lddh, a.x = x, a.ldx = ldx, a.f = f, a.ldf = ldf, a.dx = dx, a.lddx = lddx, a.df = df, a.lddf = lddf;
  a.tokens = tokens, a.channels = channels, a.starts = starts, a.s_type = s_type, a.sequences = sequences;
  a.slices = static_cast<int>(twa_ceil_div(channels, SCAN_CHANNELS));
  a.states = const_cast<float*>(static_cast<const float*>(states)), a.d_last = d_last, a.dh0 = dh0, a.status = ctx->d_status;
  int feed = scan_feed(dh, lddh, size, channels, scan_feed(f, ldf, size, channels, scan_feed(x, ldx, size, channels, BY_UNITS)));
  feed = scan_feed_out(df, lddf, size, scan_feed_out(dx, lddx, size, feed));
  TWA_CUDA_OK(ctx, dtype == TWA_BF16 ? scan_launch<bf16>(ctx, a, true, feed) : scan_launch<float>(ctx, a, true, feed));
  return TWA_OK;
}

}  // extern "C"
