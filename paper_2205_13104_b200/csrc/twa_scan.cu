// Gated linear recurrence, forward; its form, its tiles and what they cost stand in twa_scan.cuh.
//
//   h_t = a_t h_{t-1} + (1 - a_t) x_t,   a_t = sigmoid(f_t)
#include "twa_scan.cuh"

namespace {

template <typename T, int FEED, int CH>
struct ScanForward {
  typedef Place<FEED, CH> At;
  static constexpr int CHANNELS = CH;
  static constexpr int STAGES = FEED == BY_UNITS ? 3 : 2, SETS = 2;           // for which two blocks an SM have room
  static constexpr bool TOGETHER = FEED != BY_ELEMENTS;
  static constexpr int N = SEG<T>;
  static constexpr int SEGS = SCAN_CHANNELS / CH, WARP_ROWS = SEGS * N, TILE = SCAN_WARPS * WARP_ROWS;       // rows
  typedef Ring<T, FEED, CH, 2, STAGES> Rows;
  const ScanArgs& a;
  const At at;
  twa_f2 A[N], L[N];                               // of the rows up to each

  __device__ __forceinline__ ScanForward(const ScanArgs& args, int slice) : a(args), at(args, slice) {}

  __device__ __forceinline__ void row(int i, const Pair<T>& x, const Pair<T>& f) {
    const twa_f2 n = scan_gate<T>(f);
    A[i] = i ? scan_decay(n, A[i - 1]) : scan_decay(n, twa_pair(1.0f));
    L[i] = i ? scan_step(n, L[i - 1], x.both()) : scan_step(n, 0, x.both());
  }
  template <bool FULL>
  __device__ __forceinline__ void store(long long first, int rows, twa_f2 in) {
    T* h = static_cast<T*>(a.h) + first * a.ldh + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if ((FULL || i < rows) && (!TOGETHER || at.n > 0)) {
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
  // A sequence by the whole cluster.  True: `state` is the one behind it, which carry() writes.
  __device__ __forceinline__ bool whole(const Span& s, int seq, char* shared, Joins<CH / 2, SETS>& joins, Tiles<CH / 2>& tiles, int& turn, twa_f2& state) {
    Rows ring(shared, at.warp, at.lane);
    const int stride = TILE * at.ranks;
    unsigned phases = 0;
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
    state = at.state(a.h0, seq, a.channels);
    if (last_seg) joins.carry[turn ^ 1][at.pair] = state;
    int slot = scan_slot<T>(s, seq) + (at.rank * SCAN_WARPS + at.warp) * SEGS + at.seg;
    for (int t = 0; t < s.len; t += stride, slot += at.ranks * SCAN_WARPS * SEGS, h += stride * a.ldh) {
      const int first = t + at.rank * TILE + at.warp * WARP_ROWS, mine = first + at.seg * N;
      bool full = first + WARP_ROWS <= s.len;                       // the whole warp's rows exist
      int rows = scan_rows(s, mine, N);
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
        if (!share_tile<true>(a, joins, tiles, at, turn, phases, seq)) {
          rows = 0;
          full = false;
        }
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
      } else if (full) {
        store<true>(s.begin + mine, rows, in);
      } else {
        store<false>(s.begin + mine, rows, in);
      }
      ring.done();
    }
    return !scan_stopped(tiles, at.ranks) && at.rank == 0 && last_seg;
  }
  __device__ __forceinline__ void carry(int seq, twa_f2 state) const { at.keep(a.h_last, seq, a.channels, state); }

  // A sequence of at most SEG rows, by one warp: the state before each row is at hand, and rows go by, BRIEF_LOADS under way together.
  static __device__ __forceinline__ void brief(const ScanArgs& a, const At& at, const Span& s, int seq) {
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
};

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
  a.h0 = h0, a.h_last = h_last, a.states = static_cast<float*>(states), a.status = ctx->d_status, a.wait_limit_ns = ctx->wait_limit_ns, a.give_up = ctx->tune_scan_give_up;
  const int feed = scan_feed(h, ldh, size, channels, scan_feed(f, ldf, size, channels, scan_feed(x, ldx, size, channels, BY_UNITS)));
  TWA_CUDA_OK(ctx, scan_launch<ScanForward>(ctx, a, dtype, feed));
  return TWA_OK;
}

}  // extern "C"
