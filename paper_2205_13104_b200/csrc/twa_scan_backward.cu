// Gradient of the gated linear recurrence.
//
//   G_t = dh_t + a_{t+1} G_{t+1},   dx_t = (1 - a_t) G_t,   df_t = a_t (1 - a_t) (h_{t-1} - x_t) G_t
//
// Backward the states before every row are taken again from those that the forward pass kept in float32, one a segment.  What goes
// from row to row is k_t = a_t G_t, affine in the one that enters a segment from behind: k = A k_in + M with the same A as forward
// and M = sum over its rows of A_t dh_t, A_t the product of the gates up to t: both directions of a segment are taken in one pass.
#include "twa_scan.cuh"

namespace {

template <typename T, int FEED, int CH>
struct ScanBackward {
  typedef Place<FEED, CH> At;
  static constexpr int CHANNELS = CH;
  static constexpr int STAGES = 2, SETS = FEED == BY_UNITS ? 2 : 1;           // for which two blocks an SM have room
  static constexpr bool TOGETHER = FEED != BY_ELEMENTS;
  static constexpr int N = SEG<T>;
  static constexpr int SEGS = SCAN_CHANNELS / CH, WARP_ROWS = SEGS * N, TILE = SCAN_WARPS * WARP_ROWS;
  typedef Ring<T, FEED, CH, 3, STAGES> Rows;
  const ScanArgs& a;
  const At at;
  twa_f2 n[N], e[N];                               // gates; a (1 - a) (h_{t-1} - x_t)

  __device__ __forceinline__ ScanBackward(const ScanArgs& args, const At& place) : a(args), at(place) {}
  __device__ __forceinline__ ScanBackward(const ScanArgs& args, int slice) : a(args), at(args, slice) {}

  // A row on the way from the state before the segment's first row to the one behind its last; off: the segment's A and M so far.
  __device__ __forceinline__ void row(int i, const Pair<T>& x, const Pair<T>& f, const Pair<T>& dh, twa_f2& h, Map& off) {
    n[i] = scan_gate<T>(f);
    const twa_f2 d = scan_half(h, x.both()), m = twa_add2(n[i], n[i]);
    h = twa_fma2(m, d, scan_pick(n[i], h, x.both()));
    off.A = scan_decay(n[i], off.A);
    off.B = twa_fma2(off.A, dh.both(), off.B);
    float n0, n1, m0, m1;
    twa_unpair(n[i], n0, n1);
    twa_unpair(m, m0, m1);
    e[i] = twa_mul2(twa_pair(fmaf(-m0, n0, fabsf(m0)), fmaf(-m1, n1, fabsf(m1))), d);
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
  template <bool FULL, typename Dh>
  __device__ __forceinline__ void store(long long first, int rows, twa_f2& k, Dh dh) {
    T* dx = static_cast<T*>(a.dx) + (first + N - 1) * a.lddx + at.c;
    T* df = static_cast<T*>(a.df) + (first + N - 1) * a.lddf + at.c;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
      if (FULL || i < rows)
        back(i, dh(i), k, [&](float x0, float x1, float f0, float f1) {
          if (!TOGETHER || at.n > 0) {
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
  // True: `k` is the one before the sequence, which carry() writes.
  __device__ __forceinline__ bool whole(const Span& s, int seq, char* shared, Joins<CH / 2, SETS>& joins, Tiles<CH / 2>& tiles, int& turn, twa_f2& k) {
    Rows ring(shared, at.warp, at.lane);
    const int stride = TILE * at.ranks, rounds = (s.len + stride - 1) / stride;
    unsigned phases = 0;
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
    k = at.state(a.d_last, seq, a.channels);
    if (first_seg) joins.carry[turn ^ 1][at.pair] = k;
    for (int round = rounds - 1; round >= 0; --round, dx -= stride * a.lddx, df -= stride * a.lddf) {
      const int first = round * stride + at.rank * TILE + at.warp * WARP_ROWS, mine = first + at.seg * N;
      bool full = first + WARP_ROWS <= s.len;
      int rows = scan_rows(s, mine, N);
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
      if (at.seg == 0) joins.seg[turn % SETS][at.warp][at.pair] = upto;
      slot -= at.ranks * SCAN_WARPS * SEGS;
      next = round ? kept_state(at, a.states, slot, a.channels) : 0;
      __syncthreads();
      twa_f2 in;
      if (at.ranks > 1) {
        if (!share_tile<false>(a, joins, tiles, at, turn, phases, seq)) {
          rows = 0;
          full = false;
        }
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
        if (w > at.warp) in = joins.seg[turn % SETS][w][at.pair].of(in);
      if (SETS == 1) __syncthreads();
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
      } else if (full) {
        store<true>(s.begin + mine, rows, in, [&](int i) { return ring.get(2, i).both(); });
      } else {
        store<false>(s.begin + mine, rows, in, [&](int i) { return ring.get(2, i).both(); });
      }
      ring.done();
    }
    return !scan_stopped(tiles, at.ranks) && at.rank == 0 && first_seg;
  }
  __device__ __forceinline__ void carry(int seq, twa_f2 k) const { at.keep(a.dh0, seq, a.channels, k); }

  // A sequence of at most SEG rows, by one warp: the state before each row is at hand, and rows go by, BRIEF_LOADS under way together.
  static __device__ __forceinline__ void brief(const ScanArgs& a, const At& at, const Span& s, int seq) {
    const T* x = static_cast<const T*>(a.x) + s.begin * a.ldx + at.c;
    const T* f = static_cast<const T*>(a.f) + s.begin * a.ldf + at.c;
    const T* g = static_cast<const T*>(a.dh) + s.begin * a.lddh + at.c;
    ScanBackward back(a, at);
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
    back.template store<false>(s.begin, s.len, k, [&](int i) { return rd[i].both(); });
    at.keep(a.dh0, seq, a.channels, k);
  }
};

}  // namespace

extern "C" {

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
  a.states = const_cast<float*>(static_cast<const float*>(states)), a.d_last = d_last, a.dh0 = dh0, a.status = ctx->d_status, a.wait_limit_ns = ctx->wait_limit_ns, a.give_up = ctx->tune_scan_give_up;
  int feed = scan_feed(dh, lddh, size, channels, scan_feed(f, ldf, size, channels, scan_feed(x, ldx, size, channels, BY_UNITS)));
  feed = scan_feed(df, lddf, size, channels, scan_feed(dx, lddx, size, channels, feed));
  TWA_CUDA_OK(ctx, scan_launch<ScanBackward>(ctx, a, dtype, feed));
  return TWA_OK;
}

}  // extern "C"
