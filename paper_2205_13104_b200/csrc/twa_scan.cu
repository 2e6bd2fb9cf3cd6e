// Gated linear recurrence, both directions; the forms that are used here stand in twa_scan.cuh.
//
//   forward    h_t = a_t h_{t-1} + (1 - a_t) x_t,   a_t = sigmoid(f_t)
//   backward   G_t = dh_t + a_{t+1} G_{t+1},   dx_t = (1 - a_t) G_t,   df_t = a_t (1 - a_t) (h_{t-1} - x_t) G_t
//
// Backward the states before every row are taken again from those that the forward pass kept in float32, one a segment.  What goes
// from row to row is k_t = a_t G_t, affine in the one that enters a segment from behind: k = A k_in + M with the same A as forward
// and M = sum over its rows of A_t dh_t, A_t the product of the gates up to t: both directions of a segment are taken in one pass.
#include "twa_scan.cuh"

namespace {

// Affine maps v -> A v + B of two channels.
struct __align__(16) Map {
  twa_f2 A, B;
  __device__ __forceinline__ twa_f2 of(twa_f2 v) const { return twa_fma2(A, v, B); }
  __device__ __forceinline__ Map after(const Map& m) const { return {twa_mul2(A, m.A), of(m.B)}; }
};
// Of a warp's segments, joined in the order in which they are met (FORWARD: from the first): every lane's with those before its own,
// and, as `before`, those before alone.
template <bool FORWARD, int SEGS>
__device__ __forceinline__ Map join_segments(Map m, int seg, Map& before) {
  before = {twa_pair(1.0f), 0};
  if constexpr (SEGS > 1) {
    constexpr int LANES = 32 / SEGS;
    const int met = FORWARD ? seg : SEGS - 1 - seg;
    auto from = [&](const Map& v, int lanes) {
      Map r;
      r.A = FORWARD ? __shfl_up_sync(0xffffffffu, v.A, lanes) : __shfl_down_sync(0xffffffffu, v.A, lanes);
      r.B = FORWARD ? __shfl_up_sync(0xffffffffu, v.B, lanes) : __shfl_down_sync(0xffffffffu, v.B, lanes);
      return r;
    };
#pragma unroll
    for (int o = 1; o < SEGS; o *= 2) {
      const Map prev = from(m, o * LANES);
      if (met >= o) m = m.after(prev);
    }
    const Map prev = from(m, LANES);
    if (met) before = prev;
  }
  return m;
}

// What the segments of a tile make of what enters them (the state, or backward k), and what enters the next tile: twice, so that the
// next ones go beside those being read.
template <int PAIRS>
struct Joins {
  Map seg[2][SCAN_WARPS][PAIRS];
  twa_f2 carry[2][PAIRS];
};
// The same of the tiles of a cluster's blocks.
template <int PAIRS>
struct Tiles {
  Map tile[2][MAX_CLUSTER][PAIRS];
};

// The blocks of a cluster tell each other what their tiles make of a state: every warp joins its block's segments' maps, from the
// first on (FORWARD) or from the last, and the warp of each rank stores the tile's into that block.
template <bool FORWARD, int FEED, int CH>
__device__ __forceinline__ void share_tile(const Joins<CH / 2>& joins, Tiles<CH / 2>& tiles, const Place<FEED, CH>& at, int turn) {
  if (at.warp < at.ranks) {
    Map all = joins.seg[turn][FORWARD ? 0 : SCAN_WARPS - 1][at.pair];
#pragma unroll
    for (int i = 1; i < SCAN_WARPS; ++i) all = joins.seg[turn][FORWARD ? i : SCAN_WARPS - 1 - i][at.pair].after(all);
    if (at.seg == 0) {
      twa_store_remote(&tiles.tile[turn][at.rank][at.pair].A, at.warp, all.A);
      twa_store_remote(&tiles.tile[turn][at.rank][at.pair].B, at.warp, all.B);
    }
  }
  twa_cluster_sync();
}
static_assert(MAX_CLUSTER <= SCAN_WARPS, "a warp for every rank");

template <typename T, int FEED, int CH>
struct ScanForward {
  static constexpr int STAGES = 3;                 // of which two blocks an SM have room
  static constexpr bool TOGETHER = FEED != BY_ELEMENTS;
  static constexpr int N = SEG<T>;
  static constexpr int SEGS = SCAN_CHANNELS / CH, WARP_ROWS = SEGS * N, TILE = SCAN_WARPS * WARP_ROWS;       // rows
  typedef Ring<T, FEED, CH, 2, STAGES> Rows;
  const ScanArgs& a;
  const Place<FEED, CH> at;
  twa_f2 A[N], L[N];                               // of the rows up to each

  __device__ __forceinline__ ScanForward(const ScanArgs& args, const Place<FEED, CH>& place) : a(args), at(place) {}

  __device__ __forceinline__ void row(int i, const Pair<T>& x, const Pair<T>& f) {
    const twa_f2 n = scan_gate<T>(f);
    A[i] = i ? scan_decay(n, A[i - 1]) : scan_decay(n, twa_pair(1.0f));
    L[i] = i ? scan_step(n, L[i - 1], x.both()) : scan_step(n, 0, x.both());
  }
  __device__ __forceinline__ void store(long long first, int rows, twa_f2 in) {
    T* h = static_cast<T*>(a.h) + first * a.ldh + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i < rows && at.n > 0) {
        float lo, hi;
        twa_unpair(twa_fma2(A[i], in, L[i]), lo, hi);
        Pair<T>::template store<TOGETHER>(h, lo, hi, at.n);
      }
      h += a.ldh;
    }
  }
  __device__ __forceinline__ Map last(int rows) const {
    Map m = {twa_pair(1.0f), 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < rows) m = {A[i], L[i]};
    return m;
  }

  __device__ __forceinline__ void copy(Rows& ring, int array, const T* from, const void* all, long long ld, int rows) {
    const T* first = static_cast<const T*>(all);
    ring.copy(array, from, ld, rows, at.left, first, first + (a.tokens - 1) * ld + a.channels - 1);
  }
  // A sequence by the whole cluster.
  __device__ __forceinline__ void whole(const Span& s, int seq, char* shared, Joins<CH / 2>& joins, Tiles<CH / 2>& tiles, int& turn) {
    Rows ring(shared, at.warp, at.lane);
    const int stride = TILE * at.ranks;
    const bool last_seg = at.warp == SCAN_WARPS - 1 && at.seg == SEGS - 1;
    int ahead = at.rank * TILE + at.warp * WARP_ROWS;                     // row of the warp's next segments to be fetched
    ring.lies(0, static_cast<const T*>(a.x) + (s.begin + ahead) * a.ldx + at.slice, a.ldx);
    ring.lies(1, static_cast<const T*>(a.f) + (s.begin + ahead) * a.ldf + at.slice, a.ldf);
    const T* x = Rows::own(static_cast<const T*>(a.x) + (s.begin + ahead) * a.ldx + at.slice, a.ldx);
    const T* f = Rows::own(static_cast<const T*>(a.f) + (s.begin + ahead) * a.ldf + at.slice, a.ldf);
    T* h = Rows::own(static_cast<T*>(a.h) + (s.begin + ahead) * a.ldh + at.slice, a.ldh);
    auto fetch = [&]() {
      const int rows = scan_rows(s, ahead, WARP_ROWS);
      if (rows) {
        copy(ring, 0, x, a.x, a.ldx, rows);
        copy(ring, 1, f, a.f, a.ldf, rows);
      }
      ring.filled();
      ahead += stride;
      x += stride * a.ldx;
      f += stride * a.ldf;
    };
#pragma unroll
    for (int i = 0; i < Rows::AHEAD; ++i) fetch();
    twa_f2 state = at.state(a.h0, seq, a.channels);
    if (last_seg) joins.carry[turn ^ 1][at.pair] = state;
    int slot = scan_slot<T>(s, seq) + (at.rank * SCAN_WARPS + at.warp) * SEGS + at.seg;
    for (int t = 0; t < s.len; t += stride, slot += at.ranks * SCAN_WARPS * SEGS, h += stride * a.ldh) {
      const int first = t + at.rank * TILE + at.warp * WARP_ROWS, mine = first + at.seg * N;
      const bool full = first + WARP_ROWS <= s.len;                       // the whole warp's rows exist
      const int rows = scan_rows(s, mine, N);
      ring.wait();
      fetch();
      Map end;
      if (full) {
#pragma unroll
        for (int i = 0; i < N; ++i) row(i, ring.get(0, i), ring.get(1, i));
        end = {A[N - 1], L[N - 1]};
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i < rows) row(i, ring.get(0, i), ring.get(1, i));
        end = last(rows);
      }
      Map before;
      const Map upto = join_segments<true, SEGS>(end, at.seg, before);
      if (at.seg == SEGS - 1) joins.seg[turn][at.warp][at.pair] = upto;
      __syncthreads();
      twa_f2 in;
      if (at.ranks > 1) {
        share_tile<true>(joins, tiles, at, turn);
        in = state;
#pragma unroll
        for (int r = 0; r < MAX_CLUSTER; ++r) {
          const Map m = tiles.tile[turn][r][at.pair];        // at hand early; what lies behind the last rank is not used
          if (r == at.rank) in = state;
          if (r < at.ranks) state = m.of(state);
        }
      } else {
        in = joins.carry[turn ^ 1][at.pair];
      }
#pragma unroll
      for (int w = 0; w < SCAN_WARPS - 1; ++w)
        if (w < at.warp) in = joins.seg[turn][w][at.pair].of(in);
      if (SEGS > 1) in = before.of(in);
      if (rows) keep_state(at, a.states, slot, a.channels, in);
      if (at.ranks == 1 && last_seg) joins.carry[turn][at.pair] = state = end.of(in);
      turn ^= 1;
      if (FEED == BY_UNITS && full) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float lo, hi;
          twa_unpair(twa_fma2(A[i], in, L[i]), lo, hi);
          ring.put(0, i, lo, hi);
        }
        __syncwarp();
        ring.flush(0, h, a.ldh, at.left);
      } else {
        store(s.begin + mine, rows, in);
      }
      ring.done();
    }
    if (last_seg && at.rank == 0) at.keep(a.h_last, seq, a.channels, state);
  }
};

template <typename T, int FEED, int CH>
struct ScanBackward {
  static constexpr int STAGES = 2;                 // as above
  static constexpr bool TOGETHER = FEED != BY_ELEMENTS;
  static constexpr int N = SEG<T>;
  static constexpr int SEGS = SCAN_CHANNELS / CH, WARP_ROWS = SEGS * N, TILE = SCAN_WARPS * WARP_ROWS;
  typedef Ring<T, FEED, CH, 3, STAGES> Rows;
  const ScanArgs& a;
  const Place<FEED, CH> at;
  twa_f2 n[N], e[N];                               // gates; a (1 - a) (h_{t-1} - x_t)

  __device__ __forceinline__ ScanBackward(const ScanArgs& args, const Place<FEED, CH>& place) : a(args), at(place) {}

  // A row on the way from the state before the segment's first row to the one behind its last; off: the segment's A and M so far.
  __device__ __forceinline__ void row(int i, const Pair<T>& x, const Pair<T>& f, const Pair<T>& dh, twa_f2& h, Map& off) {
    n[i] = scan_gate<T>(f);
    const twa_f2 d = scan_minus(h, x.both());
    h = twa_fma2(n[i], d, scan_pick(n[i], h, x.both()));
    off.A = scan_decay(n[i], off.A);
    off.B = twa_fma2(off.A, dh.both(), off.B);
    float n0, n1;
    twa_unpair(n[i], n0, n1);
    e[i] = twa_mul2(twa_pair(fmaf(-n0, n0, fabsf(n0)), fmaf(-n1, n1, fabsf(n1))), d);
  }
  // Gradients of a row from g = dh + k, where k is what comes from the rows behind it; k becomes this row's.  With p = n g, k is
  // g + p where the gate is open and p where not, and dx = (1 - a) g is -p or g - p.
  template <typename Out>
  __device__ __forceinline__ void back(int i, twa_f2 dh, twa_f2& k, Out out) {
    const twa_f2 g = twa_add2(dh, k), p = twa_mul2(n[i], g), open = scan_pick(n[i], g, twa_pair(0.0f));
    k = twa_add2(open, p);
    float x0, x1, f0, f1;
    twa_unpair(scan_minus(scan_minus(g, open), p), x0, x1);
    twa_unpair(twa_mul2(e[i], g), f0, f1);
    out(x0, x1, f0, f1);
  }
  // Of the first `rows` rows from `first` on, straight to memory.
  template <typename Dh>
  __device__ __forceinline__ void store(long long first, int rows, twa_f2& k, Dh dh) {
    T* dx = static_cast<T*>(a.dx) + (first + N - 1) * a.lddx + at.c;
    T* df = static_cast<T*>(a.df) + (first + N - 1) * a.lddf + at.c;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
      if (i < rows)
        back(i, dh(i), k, [&](float x0, float x1, float f0, float f1) {
          if (at.n > 0) {
            Pair<T>::template store<TOGETHER>(dx, x0, x1, at.n);
            Pair<T>::template store<TOGETHER>(df, f0, f1, at.n);
          }
        });
      dx -= a.lddx;
      df -= a.lddf;
    }
  }

  __device__ __forceinline__ void copy(Rows& ring, int array, const T* from, const void* all, long long ld, int rows) {
    const T* first = static_cast<const T*>(all);
    ring.copy(array, from, ld, rows, at.left, first, first + (a.tokens - 1) * ld + a.channels - 1);
  }
  __device__ __forceinline__ void whole(const Span& s, int seq, char* shared, Joins<CH / 2>& joins, Tiles<CH / 2>& tiles, int& turn) {
    Rows ring(shared, at.warp, at.lane);
    const int stride = TILE * at.ranks, rounds = (s.len + stride - 1) / stride;
    const bool first_seg = at.warp == 0 && at.seg == 0;
    int ahead = (rounds - 1) * stride + at.rank * TILE + at.warp * WARP_ROWS;
    ring.lies(0, static_cast<const T*>(a.x) + (s.begin + ahead) * a.ldx + at.slice, a.ldx);
    ring.lies(1, static_cast<const T*>(a.f) + (s.begin + ahead) * a.ldf + at.slice, a.ldf);
    ring.lies(2, static_cast<const T*>(a.dh) + (s.begin + ahead) * a.lddh + at.slice, a.lddh);
    const T* x = Rows::own(static_cast<const T*>(a.x) + (s.begin + ahead) * a.ldx + at.slice, a.ldx);
    const T* f = Rows::own(static_cast<const T*>(a.f) + (s.begin + ahead) * a.ldf + at.slice, a.ldf);
    const T* g = Rows::own(static_cast<const T*>(a.dh) + (s.begin + ahead) * a.lddh + at.slice, a.lddh);
    T* dx = Rows::own(static_cast<T*>(a.dx) + (s.begin + ahead) * a.lddx + at.slice, a.lddx);
    T* df = Rows::own(static_cast<T*>(a.df) + (s.begin + ahead) * a.lddf + at.slice, a.lddf);
    // the state before the next segment, fetched one tile ahead
    int slot = scan_slot<T>(s, seq) + ((rounds - 1) * at.ranks + at.rank) * SCAN_WARPS * SEGS + at.warp * SEGS + at.seg;
    twa_f2 next = rounds && ahead + at.seg * N < s.len ? kept_state(at, a.states, slot, a.channels) : 0;
    auto fetch = [&]() {
      const int rows = ahead < 0 ? 0 : scan_rows(s, ahead, WARP_ROWS);
      if (rows) {
        copy(ring, 0, x, a.x, a.ldx, rows);
        copy(ring, 1, f, a.f, a.ldf, rows);
        copy(ring, 2, g, a.dh, a.lddh, rows);
      }
      ring.filled();
      ahead -= stride;
      x -= stride * a.ldx;
      f -= stride * a.ldf;
      g -= stride * a.lddh;
    };
#pragma unroll
    for (int i = 0; i < Rows::AHEAD; ++i) fetch();
    twa_f2 k = at.state(a.d_last, seq, a.channels);
    if (first_seg) joins.carry[turn ^ 1][at.pair] = k;
    for (int round = rounds - 1; round >= 0; --round, dx -= stride * a.lddx, df -= stride * a.lddf) {
      const int first = round * stride + at.rank * TILE + at.warp * WARP_ROWS, mine = first + at.seg * N;
      const bool full = first + WARP_ROWS <= s.len;
      const int rows = scan_rows(s, mine, N);
      twa_f2 h = next;
      ring.wait();
      fetch();
      Map off = {twa_pair(1.0f), 0};
      if (full) {
#pragma unroll
        for (int i = 0; i < N; ++i) row(i, ring.get(0, i), ring.get(1, i), ring.get(2, i), h, off);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i < rows) row(i, ring.get(0, i), ring.get(1, i), ring.get(2, i), h, off);
      }
      Map behind;
      const Map upto = join_segments<false, SEGS>(off, at.seg, behind);
      if (at.seg == 0) joins.seg[turn][at.warp][at.pair] = upto;
      slot -= at.ranks * SCAN_WARPS * SEGS;
      next = round ? kept_state(at, a.states, slot, a.channels) : 0;
      __syncthreads();
      twa_f2 in;
      if (at.ranks > 1) {
        share_tile<false>(joins, tiles, at, turn);
        in = k;
#pragma unroll
        for (int r = MAX_CLUSTER - 1; r >= 0; --r) {
          const Map m = tiles.tile[turn][r][at.pair];
          if (r == at.rank) in = k;
          if (r < at.ranks) k = m.of(k);
        }
      } else {
        in = joins.carry[turn ^ 1][at.pair];
      }
#pragma unroll
      for (int w = SCAN_WARPS - 1; w > 0; --w)
        if (w > at.warp) in = joins.seg[turn][w][at.pair].of(in);
      if (SEGS > 1) in = behind.of(in);
      if (at.ranks == 1 && first_seg) joins.carry[turn][at.pair] = k = off.of(in);
      turn ^= 1;
      if (FEED == BY_UNITS && full) {
#pragma unroll
        for (int i = N - 1; i >= 0; --i)
          back(i, ring.get(2, i).both(), in, [&](float x0, float x1, float f0, float f1) {
            ring.put(0, i, x0, x1);
            ring.put(1, i, f0, f1);
          });
        __syncwarp();
        ring.flush(0, dx, a.lddx, at.left);
        ring.flush(1, df, a.lddf, at.left);
      } else {
        store(s.begin + mine, rows, in, [&](int i) { return ring.get(2, i).both(); });
      }
      ring.done();
    }
    if (first_seg && at.rank == 0) at.keep(a.dh0, seq, a.channels, k);
  }
};

// A sequence of at most SEG rows, by one warp: the state before each row is at hand, and rows go by, BRIEF_LOADS under way together.
constexpr int BRIEF_LOADS = 4;
template <typename T, int FEED>
__device__ __forceinline__ void brief_forward(const ScanArgs& a, const Place<FEED, SCAN_CHANNELS>& at, const Span& s, int seq) {
  constexpr bool TOGETHER = FEED != BY_ELEMENTS;
  const T* x = static_cast<const T*>(a.x) + s.begin * a.ldx + at.c;
  const T* f = static_cast<const T*>(a.f) + s.begin * a.ldf + at.c;
  T* h = static_cast<T*>(a.h) + s.begin * a.ldh + at.c;
  twa_f2 state = 0;
  for (int r = 0; r < s.len; r += BRIEF_LOADS) {
    Pair<T> rx[BRIEF_LOADS], rf[BRIEF_LOADS];
#pragma unroll
    for (int i = 0; i < BRIEF_LOADS; ++i)
      if (r + i < s.len && at.n > 0) {
        rx[i].template load<TOGETHER>(x + (r + i) * a.ldx, at.n);
        rf[i].template load<TOGETHER>(f + (r + i) * a.ldf, at.n);
      }
    if (r == 0) {
      state = at.state(a.h0, seq, a.channels);
      keep_state(at, a.states, scan_slot<T>(s, seq), a.channels, state);
    }
#pragma unroll
    for (int i = 0; i < BRIEF_LOADS; ++i)
      if (r + i < s.len && at.n > 0) {
        state = scan_step(scan_gate<T>(rf[i]), state, rx[i].both());
        float lo, hi;
        twa_unpair(state, lo, hi);
        Pair<T>::template store<TOGETHER>(h + (r + i) * a.ldh, lo, hi, at.n);
      }
  }
  if (s.len == 0) state = at.state(a.h0, seq, a.channels);
  at.keep(a.h_last, seq, a.channels, state);
}
template <typename T, int FEED>
__device__ __forceinline__ void brief_backward(const ScanArgs& a, const Place<FEED, SCAN_CHANNELS>& at, const Span& s, int seq) {
  constexpr bool TOGETHER = FEED != BY_ELEMENTS;
  const T* x = static_cast<const T*>(a.x) + s.begin * a.ldx + at.c;
  const T* f = static_cast<const T*>(a.f) + s.begin * a.ldf + at.c;
  const T* g = static_cast<const T*>(a.dh) + s.begin * a.lddh + at.c;
  ScanBackward<T, FEED, SCAN_CHANNELS> back(a, at);
  constexpr int N = SEG<T>;
  Pair<T> rd[N];
  twa_f2 h = s.len ? kept_state(at, a.states, scan_slot<T>(s, seq), a.channels) : 0;
  twa_f2 k = at.state(a.d_last, seq, a.channels);
  Map off = {twa_pair(1.0f), 0};
#pragma unroll
  for (int r = 0; r < N; r += BRIEF_LOADS)
    if (r < s.len) {
      Pair<T> rx[BRIEF_LOADS], rf[BRIEF_LOADS];
#pragma unroll
      for (int i = 0; i < BRIEF_LOADS; ++i)
        if (r + i < s.len && at.n > 0) {
          rx[i].template load<TOGETHER>(x + (r + i) * a.ldx, at.n);
          rf[i].template load<TOGETHER>(f + (r + i) * a.ldf, at.n);
          rd[r + i].template load<TOGETHER>(g + (r + i) * a.lddh, at.n);
        }
#pragma unroll
      for (int i = 0; i < BRIEF_LOADS; ++i)
        if (r + i < s.len) back.row(r + i, rx[i], rf[i], rd[r + i], h, off);
    }
  back.store(s.begin, s.len, k, [&](int i) { return rd[i].both(); });
  at.keep(a.dh0, seq, a.channels, k);
}
template <typename T, int FEED, bool BACK>
__device__ __forceinline__ void scan_brief(const ScanArgs& a, const Place<FEED, SCAN_CHANNELS>& at, const Span& s, int seq) {
  if constexpr (BACK) brief_backward<T, FEED>(a, at, s, seq);
  else brief_forward<T, FEED>(a, at, s, seq);
}
// Where no sequence is longer: a warp for each, of each slice.
template <typename T, int FEED, bool BACK>
__global__ void __launch_bounds__(SCAN_THREADS) scan_brief_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.dh, a.h0, a.states, a.d_last);
  const int slice = blockIdx.x % a.slices, seq = blockIdx.x / a.slices * SHORT_GROUP + (threadIdx.x >> 5);
  const Place<FEED, SCAN_CHANNELS> at(a, slice);
  if (seq < a.sequences) scan_brief<T, FEED, BACK>(a, at, scan_span(a, seq, false), seq);
}

// GROUP sequences of a slice of channels a block.  The ones of at most SEG rows go to one warp each, the others to the block.
template <typename Direction, typename T, int FEED, bool BACK, int CH, int GROUP>
__device__ __forceinline__ void scan_block(const ScanArgs& a) {
  extern __shared__ __align__(16) char shared[];
  __shared__ Joins<CH / 2> joins;
  Tiles<CH / 2>& tiles = *reinterpret_cast<Tiles<CH / 2>*>(shared + Direction::Rows::BLOCK_BYTES);         // of clusters only
  const unsigned task = blockIdx.x / a.cluster;
  const int slice = task % a.slices, first = task / a.slices * GROUP;
  Direction d(a, Place<FEED, CH>(a, slice));
  if (a.cluster > 1) twa_cluster_sync();           // no block stores into one that has not begun
  if constexpr (GROUP > 1) {
    const int seq = first + d.at.warp;
    if (seq < a.sequences) {
      const Span s = scan_span(a, seq, slice == 0 && d.at.lane == 0);
      if (s.len >= 0 && s.len <= Direction::N) scan_brief<T, FEED, BACK>(a, d.at, s, seq);
    }
  }
  int turn = 0;
  for (int g = 0; g < GROUP; ++g) {
    const int seq = first + g;
    if (seq >= a.sequences) break;
    const Span s = scan_span(a, seq, GROUP == 1 && slice == 0 && threadIdx.x == 0);
    if (s.len > Direction::N || (GROUP == 1 && s.len >= 0)) d.whole(s, seq, shared, joins, tiles, turn);
  }
}

template <typename T, int FEED, int CH, int GROUP>
__global__ void __launch_bounds__(SCAN_THREADS, 2) scan_forward_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.starts, a.h0);
  scan_block<ScanForward<T, FEED, CH>, T, FEED, false, CH, GROUP>(a);
}
template <typename T, int FEED, int CH, int GROUP>
__global__ void __launch_bounds__(SCAN_THREADS, 2) scan_backward_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.dh, a.starts, a.states, a.d_last);
  scan_block<ScanBackward<T, FEED, CH>, T, FEED, true, CH, GROUP>(a);
}

// How rows of two pointers and strides can be fetched together.
int scan_feed(const void* p, long long ld, size_t size, int channels, int so_far) {
  if (so_far == BY_UNITS && (channels * size % 16 || twa_misaligned_to(p, 16) || ld * size % 16)) so_far = BY_PAIRS;
  if (so_far == BY_PAIRS && (channels % 2 || twa_misaligned_to(p, 2 * size) || ld % 2)) so_far = BY_ELEMENTS;
  return so_far;
}
template <typename T, int FEED, int CH, int GROUP>
cudaError_t scan_launch(twa_ctx* ctx, const ScanArgs& a, bool back) {
  auto kernel = back ? scan_backward_kernel<T, FEED, CH, GROUP> : scan_forward_kernel<T, FEED, CH, GROUP>;
  const size_t smem = (back ? ScanBackward<T, FEED, CH>::Rows::BLOCK_BYTES : ScanForward<T, FEED, CH>::Rows::BLOCK_BYTES) + (a.cluster > 1 ? sizeof(Tiles<CH / 2>) : 0);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.sequences, GROUP) * a.slices * a.cluster);
  return twa_launch_clusters(ctx->stream, kernel, blocks, a.cluster, SCAN_THREADS, smem, a);
}
constexpr int SCAN_RESIDENT = 2;                   // blocks of an SM
template <typename T>
cudaError_t scan_launch(twa_ctx* ctx, ScanArgs& a, bool back, int feed) {
  a.cluster = 1;
  // A warp a sequence: all of them where they are short enough, or, of ragged ones, those that are, where most must be.
  const bool short_all = !a.starts && a.tokens <= static_cast<long long>(SEG<T>) * a.sequences;
  if (short_all || (a.starts && 2 * a.tokens <= static_cast<long long>(SEG<T>) * a.sequences)) {
    a.slices = static_cast<int>(twa_ceil_div(a.channels, SCAN_CHANNELS));
    if (short_all) {
      const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.sequences, SHORT_GROUP) * a.slices);
      auto launch = [&](auto kernel) { return twa_launch(ctx->stream, kernel, blocks, SCAN_THREADS, 0, a); };
      if (back) return feed == BY_ELEMENTS ? launch(scan_brief_kernel<T, BY_ELEMENTS, true>) : launch(scan_brief_kernel<T, BY_PAIRS, true>);
      return feed == BY_ELEMENTS ? launch(scan_brief_kernel<T, BY_ELEMENTS, false>) : launch(scan_brief_kernel<T, BY_PAIRS, false>);
    }
    return feed == BY_UNITS ? scan_launch<T, BY_UNITS, SCAN_CHANNELS, SHORT_GROUP>(ctx, a, back)
                            : (feed == BY_PAIRS ? scan_launch<T, BY_PAIRS, SCAN_CHANNELS, SHORT_GROUP>(ctx, a, back)
                                                : scan_launch<T, BY_ELEMENTS, SCAN_CHANNELS, SHORT_GROUP>(ctx, a, back));
  }
  int channels = SCAN_CHANNELS;
  auto blocks = [&]() { return twa_ceil_div(a.channels, channels) * a.sequences * a.cluster; };
  auto rows = [&]() { return a.cluster * SCAN_WARPS * SEG<T> * (SCAN_CHANNELS / channels); };       // of a round
  // Twice as many where there is room for them and rows enough; ragged sequences wait for the longest, which takes the more blocks
  // (15 ragged sequences of 13138 x 1016 bfloat16, both directions 133 us with one block each, 110 with two).
  const int places = (a.starts ? 2 : 1) * SCAN_RESIDENT * ctx->sm_count;
  auto more = [&]() { return 2 * blocks() <= places && a.tokens > 2LL * rows() * a.sequences; };
  if (ctx->tune_scan_channels && feed == BY_UNITS) channels = ctx->tune_scan_channels;
  else if (feed == BY_UNITS && more()) channels = 32;
  while (a.cluster < MAX_CLUSTER && more()) a.cluster *= 2;
  if (!ctx->tune_scan_channels && channels == 32 && more()) channels = 16;
  if (ctx->tune_scan_cluster) a.cluster = ctx->tune_scan_cluster;
  a.slices = static_cast<int>(twa_ceil_div(a.channels, channels));
  if (feed == BY_PAIRS) return scan_launch<T, BY_PAIRS, SCAN_CHANNELS, 1>(ctx, a, back);
  if (feed == BY_ELEMENTS) return scan_launch<T, BY_ELEMENTS, SCAN_CHANNELS, 1>(ctx, a, back);
  return channels == 64 ? scan_launch<T, BY_UNITS, 64, 1>(ctx, a, back)
                        : (channels == 32 ? scan_launch<T, BY_UNITS, 32, 1>(ctx, a, back) : scan_launch<T, BY_UNITS, 16, 1>(ctx, a, back));
}

// Arguments that both directions have.
int scan_check(twa_ctx* ctx, int dtype, int64_t tokens, int channels, const void* starts, int s_type, int sequences) {
  if (!ctx || !twa_dtype_ok(dtype) || tokens < 0 || channels < 1 || sequences < 0 || (starts && !twa_itype_ok(s_type))) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_SCAN_MAX_TOKENS || channels > TWA_SCAN_MAX_CHANNELS || sequences > TWA_SCAN_MAX_SEQUENCES) return TWA_ERR_UNSUPPORTED;
  if (!starts && (sequences ? tokens % sequences : tokens)) return TWA_ERR_INVALID_ARG;
  if (starts && twa_misaligned_to(starts, twa_itype_size(s_type))) return TWA_ERR_MISALIGNED;
  // blocks of a launch
  if (static_cast<long long>(sequences) * twa_ceil_div(channels, SCAN_LEAST_CHANNELS) * MAX_CLUSTER > 0x7FFFFFFFLL) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

}  // namespace

extern "C" {

size_t twa_gated_scan_states_bytes(int64_t tokens, int sequences, int channels) {
  if (tokens < 0 || tokens > TWA_SCAN_MAX_TOKENS || sequences < 0 || sequences > TWA_SCAN_MAX_SEQUENCES || channels < 1 ||
      channels > TWA_SCAN_MAX_CHANNELS)
    return 0;
  return static_cast<size_t>(tokens / STATE_ROWS + sequences) * channels * sizeof(float);
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
  a.h0 = h0, a.h_last = h_last, a.states = static_cast<float*>(states), a.status = ctx->d_status;
  const int feed = scan_feed(h, ldh, size, channels, scan_feed(f, ldf, size, channels, scan_feed(x, ldx, size, channels, BY_UNITS)));
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
  a.states = const_cast<float*>(static_cast<const float*>(states)), a.d_last = d_last, a.dh0 = dh0, a.status = ctx->d_status;
  int feed = scan_feed(dh, lddh, size, channels, scan_feed(f, ldf, size, channels, scan_feed(x, ldx, size, channels, BY_UNITS)));
  feed = scan_feed(df, lddf, size, channels, scan_feed(dx, lddx, size, channels, feed));
  TWA_CUDA_OK(ctx, dtype == TWA_BF16 ? scan_launch<bf16>(ctx, a, true, feed) : scan_launch<float>(ctx, a, true, feed));
  return TWA_OK;
}

}  // extern "C"
