// Gated linear recurrence: what its two directions share.
//
//   a_t = sigmoid(f_t),   h_t = a_t h_{t-1} + (1 - a_t) x_t          for every channel of every sequence
//
// A step is taken from the smaller of a and 1 - a, s = 1 / (1 + e^|f|), which keeps its digits however near one the other is:
//   f >= 0 (s = 1 - a):  h' = h + s (x - h)        f < 0 (s = a):  h' = x + s (h - x) = x - s (x - h)
// or, with q = s under the sign of f, h' = q (x - h) + (f >= 0 ? h : x): one subtraction and one fused product, whose rounding
// is half a unit of the result; a gate rounded to 1 - 2^-24 k would err the same way step after step.  Steps in a row are
// affine in the state that enters, h = A h_in + L; A comes from the same steps with x = 0 from 1, L with h_in = 0.
//
// A lane has two channels and SEG rows of them, a segment, which it takes from 0.  A slice of 64 channels gives every warp one
// segment, one of 32 or 16 two or four, a lane's neighbours in other segments; the segments of a block follow each other and are its
// tile.  A warp joins its segments' (A, L) by shuffles, the warps' go through shared memory, and every thread joins those before its
// own with the state that enters the tile.  States are float32.
//
// One pass over x and f (and dh), which come through a ring of asynchronous copies, and one store.  Blocks differ in sequence and
// slice; where those are few a cluster of blocks takes a sequence together, a tile each a round, and tells each other what the tiles
// make of a state.  Everything is joined in a fixed order: results repeat bit for bit.
// With equal blocks in every place the bound is memory: 2 x 8192 x 9472 bfloat16 forward, 296 of them, 153 us for 931 MB (6.1 TB/s).
// 8 x 2048 x 2048 bfloat16: 42 us forward (201 MB, floor 31) and 61 backward (335 MB, 52).  256 blocks for 296 places are a factor of
// 1.16; the rest is latency: DRAM at 45 and 57 % of its peak and issue slots at 55 and 59 %, while two blocks of 8 warps an SM, 128
// registers each, are all there is to hide the copies' wait, the steps that follow one another, the barrier and the joins.
// Where a round's latency counts: 1 x 65536 x 512 float32 99 and 139 us (floors 62 and 104).  (Calls in a row, inputs from DRAM.)
// A lane's rows are as many as its registers hold between the two passes over them (their A and L): 8 rows of bfloat16 a lane and three
// blocks an SM instead of 16 and two took 55 and 86 us for 47 and 68 (single calls), as the joins are paid once a tile; slices of 56 channels, which
// give 296 blocks, 55 and 82, as rows of 112 bytes share sectors.  Plain instead of packed arithmetic cost 24 instead of 21
// instructions an element forward and the same time.
#pragma once

#include "twa_ops.cuh"

namespace {

constexpr int SCAN_WARPS = 8, SCAN_THREADS = SCAN_WARPS * 32;
template <typename T>
constexpr int SEG = 32 / sizeof(T);                // rows of a segment
constexpr int STATE_ROWS = SEG<float>;             // from one kept state to the next, at least
constexpr int SCAN_CHANNELS = 64, SCAN_LEAST_CHANNELS = 16;               // of a block, at most and at least
constexpr int SHORT_GROUP = SCAN_WARPS;            // sequences of a block where most are short
constexpr int BRIEF_LOADS = 4;                     // rows of a short sequence under way together
constexpr int MAX_CLUSTER = 8;                     // blocks along a sequence

struct ScanArgs {
  const void *x, *f, *dh;
  void *h, *dx, *df;
  long long ldx, ldf, lddh, ldh, lddx, lddf;
  long long tokens;
  const void* starts;
  int s_type, sequences, channels, slices, cluster;
  bool by_length;                                  // ragged sequences, the longest first
  const float* h0;
  float* h_last;
  float* states;
  const float* d_last;
  float* dh0;
  int* status;
  unsigned long long wait_limit_ns;
  int give_up;                                     // 1 + 8 x rank + warp: which takes its wait for one that ran out (0: none)
};

// Rows of a sequence; len -1: its offsets are wrong and it is left alone.
struct Span {
  long long begin;
  int len;
};
template <bool RAGGED>
__device__ __forceinline__ Span scan_span(const ScanArgs& a, int seq, bool report) {
  if (!RAGGED) {
    const int each = static_cast<int>(a.tokens / a.sequences);
    return {static_cast<long long>(seq) * each, each};
  }
  const long long b = twa_load_id(a.starts, a.s_type, seq), e = twa_load_id(a.starts, a.s_type, seq + 1);
  if (b < 0 || e < b || e > a.tokens) {
    if (report) twa_set_status(a.status, TWA_ERR_INVALID_ARG, seq);
    return {0, -1};
  }
  return {b, static_cast<int>(e - b)};
}
// The first of a sequence's kept states: those of sequences before it end before this place, for
// (b + len) / R + 1 >= b / R + ceil(len / R).
template <typename T>
__device__ __forceinline__ int scan_slot(const Span& s, int seq) { return static_cast<int>(s.begin / SEG<T>) + seq; }
// Rows that a sequence has from row r on, of `most`.
__device__ __forceinline__ int scan_rows(const Span& s, int r, int most) { return min(max(s.len - r, 0), most); }

// How rows lie, and which two channels a lane has.  In units of 16 bytes: neighbours; rows are copied and stored by the unit, any
// lane's.  In pairs: neighbours, stored together.  Element by element, where rows lie on no such boundary: channels 32 apart, so
// that a warp's accesses are contiguous.
enum { BY_UNITS, BY_PAIRS, BY_ELEMENTS };

// Stores an element where `exists`: a predicate, no branch.
template <int OFFSET>
__device__ __forceinline__ void scan_store(float* p, uint32_t v, bool exists) {
  asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %2, 0;\n@q st.global.b32 [%0 + %3], %1;\n}" ::"l"(p), "r"(v), "r"(static_cast<int>(exists)), "n"(OFFSET)
               : "memory");
}
template <int OFFSET>
__device__ __forceinline__ void scan_store(bf16* p, unsigned short v, bool exists) {
  asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %2, 0;\n@q st.global.b16 [%0 + %3], %1;\n}" ::"l"(p), "h"(v), "r"(static_cast<int>(exists)), "n"(OFFSET)
               : "memory");
}

// Two elements in one or two registers.
template <typename T>
struct Pair;
template <>
struct Pair<float> {
  float2 r;
  template <bool TOGETHER>
  __device__ __forceinline__ void load(const float* p, int n) {
    if constexpr (TOGETHER) r = __ldg(reinterpret_cast<const float2*>(p));
    else {
      r.x = __ldg(p);
      r.y = n > 1 ? __ldg(p + 32) : 0.0f;
    }
  }
  __device__ __forceinline__ float lo() const { return r.x; }
  __device__ __forceinline__ float hi() const { return r.y; }
  __device__ __forceinline__ twa_f2 both() const { return twa_pair(r.x, r.y); }
  template <bool TOGETHER>
  static __device__ __forceinline__ void store(float* p, float a, float b, int n) {
    if constexpr (TOGETHER) *reinterpret_cast<float2*>(p) = make_float2(a, b);
    else {
      scan_store<0>(p, __float_as_uint(a), n > 0);
      scan_store<128>(p, __float_as_uint(b), n > 1);
    }
  }
};
template <>
struct Pair<bf16> {
  uint32_t r;
  template <bool TOGETHER>
  __device__ __forceinline__ void load(const bf16* p, int n) {
    if constexpr (TOGETHER) r = __ldg(reinterpret_cast<const uint32_t*>(p));
    else {
      const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
      r = __ldg(q);
      if (n > 1) r |= static_cast<uint32_t>(__ldg(q + 32)) << 16;
    }
  }
  __device__ __forceinline__ float lo() const { return twa_bf16_lo(r); }
  __device__ __forceinline__ float hi() const { return twa_bf16_hi(r); }
  __device__ __forceinline__ twa_f2 both() const { return twa_pair(lo(), hi()); }
  template <bool TOGETHER>
  static __device__ __forceinline__ void store(bf16* p, float a, float b, int n) {
    if constexpr (TOGETHER) *reinterpret_cast<uint32_t*>(p) = twa_bf16_pair(a, b);
    else {
      scan_store<0>(p, __bfloat16_as_ushort(twa_from_float<bf16>(a)), n > 0);
      scan_store<64>(p, __bfloat16_as_ushort(twa_from_float<bf16>(b)), n > 1);
    }
  }
};

// -q of two gates; their signs say which form a step takes.  1 + e^|f|: the exponential of a bfloat16 gate may err by some units of
// float32 and is taken as a power of two at once, both exponents by one product; that of a float32 gate may not.
__device__ __forceinline__ float scan_exp2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fabsf(v)));
  return r;
}
__device__ __forceinline__ twa_f2 scan_exp(const Pair<float>& f) { return twa_pair(expf(fabsf(f.lo())), expf(fabsf(f.hi()))); }
__device__ __forceinline__ twa_f2 scan_exp(const Pair<bf16>& f) {
  float a, b;
  twa_unpair(twa_mul2(f.both(), twa_pair(1.44269504f)), a, b);
  return twa_pair(scan_exp2(a), scan_exp2(b));
}
__device__ __forceinline__ float scan_reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float scan_turn(float s, float f) {
  return __uint_as_float(__float_as_uint(s) | (~__float_as_uint(f) & 0x80000000u));
}
template <typename T>
__device__ __forceinline__ twa_f2 scan_gate(const Pair<T>& f) {
  float a, b;
  twa_unpair(twa_add2(twa_pair(1.0f), scan_exp(f)), a, b);
  return twa_pair(scan_turn(scan_reciprocal(a), f.lo()), scan_turn(scan_reciprocal(b), f.hi()));
}
__device__ __forceinline__ bool scan_open(float n) { return __float_as_int(n) < 0; }
// (open ? a : b) of two gates.
__device__ __forceinline__ twa_f2 scan_pick(twa_f2 n, twa_f2 a, twa_f2 b) {
  float n0, n1, a0, a1, b0, b1;
  twa_unpair(n, n0, n1);
  twa_unpair(a, a0, a1);
  twa_unpair(b, b0, b1);
  return twa_pair(scan_open(n0) ? a0 : b0, scan_open(n1) ? a1 : b1);
}
__device__ __forceinline__ twa_f2 scan_minus(twa_f2 a, twa_f2 b) { return twa_fma2(b, twa_pair(-1.0f), a); }
// Half of h - x, which twice a gate is multiplied with: two finite values may be further apart than the largest float32.  Halves and
// doubles have the digits of the whole (but for the last ones of numbers next to the smallest).
__device__ __forceinline__ twa_f2 scan_half(twa_f2 h, twa_f2 x) { return twa_fma2(h, twa_pair(0.5f), twa_mul2(x, twa_pair(-0.5f))); }
__device__ __forceinline__ twa_f2 scan_step(twa_f2 n, twa_f2 h, twa_f2 x) { return twa_fma2(twa_add2(n, n), scan_half(h, x), scan_pick(n, h, x)); }
// a times v: what a step makes of a state where x is 0.
__device__ __forceinline__ twa_f2 scan_decay(twa_f2 n, twa_f2 v) { return twa_fma2(n, v, scan_pick(n, v, twa_pair(0.0f))); }

// A value that is the same for the whole warp, in a register of the warp's: addresses and counts that follow from it cost a lane nothing.
__device__ __forceinline__ int uniform(int v) { return static_cast<int>(__reduce_max_sync(0xffffffffu, static_cast<unsigned>(v))); }

// Where a thread stands: its two channels, c and c + 1 or c and c + 32, of which n exist; which of its warp's segments it has, and which
// pair of the segment's channels; its block's rank along the sequence.
template <int FEED, int CH>
struct Place {
  static constexpr int NEXT = FEED == BY_ELEMENTS ? 32 : 1, SEGS = SCAN_CHANNELS / CH, PAIRS = CH / 2;
  int lane, warp, slice, left, seg, pair, c, n, rank, ranks;      // left: channels of the slice
  __device__ __forceinline__ Place(const ScanArgs& a, int part) {
    lane = threadIdx.x & 31;
    warp = uniform(threadIdx.x >> 5);
    slice = part * CH;
    left = min(CH, a.channels - slice);
    seg = SEGS > 1 ? lane / PAIRS : 0;
    pair = SEGS > 1 ? lane % PAIRS : lane;
    c = slice + (FEED == BY_ELEMENTS ? lane : 2 * pair);
    n = (c < a.channels ? 1 : 0) + (c + NEXT < a.channels ? 1 : 0);
    ranks = a.cluster;
    rank = ranks > 1 ? static_cast<int>(twa_cluster_rank()) : 0;
  }
  // Its channels of a row of float32 states.
  __device__ __forceinline__ twa_f2 state(const float* p, long long row, int channels) const {
    if (!p) return 0;
    return twa_pair(n > 0 ? p[row * channels + c] : 0.0f, n > 1 ? p[row * channels + c + NEXT] : 0.0f);
  }
  __device__ __forceinline__ void keep(float* p, long long row, int channels, twa_f2 v) const {
    if (!p) return;
    float lo, hi;
    twa_unpair(v, lo, hi);
    if (n > 0) p[row * channels + c] = lo;
    if (n > 1) p[row * channels + c + NEXT] = hi;
  }
};

// The states that the forward pass keeps: the same, but the buffer is the library's and begins on 16 bytes.
template <int FEED, int CH>
__device__ __forceinline__ twa_f2 kept_state(const Place<FEED, CH>& at, const float* p, long long row, int channels) {
  if (FEED == BY_ELEMENTS) return at.state(p, row, channels);
  twa_f2 v = 0;
  if (at.n > 0) v = *reinterpret_cast<const twa_f2*>(p + row * channels + at.c);
  return v;
}
template <int FEED, int CH>
__device__ __forceinline__ void keep_state(const Place<FEED, CH>& at, float* p, long long row, int channels, twa_f2 v) {
  if (FEED == BY_ELEMENTS) at.keep(p, row, channels, v);
  else if (p && at.n > 0) *reinterpret_cast<twa_f2*>(p + row * channels + at.c) = v;
}

// A ring of a warp's segments in shared memory, STAGES deep, of ARRAYS matrices, filled by asynchronous copies.  A segment begins a
// row's length behind the one before it, so that lanes of different segments read different banks.  By units, results go
// out the same way: pairs into the stage that has been read, and from there 16 bytes a lane.
// Rows that are not in units come in the 16-byte pieces in which they lie, one more than a row has, and elements are found from where
// the row begins in its first piece; a piece that reaches out of the matrix is filled by the element.  (Copies of the 4-byte words,
// or of the pairs, were four times as many: 37 ragged sequences of 20011 x 771 bfloat16 67 and 101 us, so 53 and 82.)
template <typename T, int FEED, int CH, int ARRAYS, int STAGES>
struct Ring {
  static constexpr int N = SEG<T>, SEGS = SCAN_CHANNELS / CH;
  static_assert(SEGS == 1 || FEED == BY_UNITS, "narrow slices by units only");
  static constexpr bool PIECES = FEED != BY_UNITS;
  static constexpr int ROW = CH * sizeof(T) + (PIECES ? 16 : 0), NEXT_SEG = (N + (SEGS > 1 ? 1 : 0)) * ROW;       // bytes
  static constexpr int AREA = SEGS * NEXT_SEG, BYTES = ARRAYS * AREA;                                            // of a matrix, a stage
  static constexpr size_t BLOCK_BYTES = static_cast<size_t>(SCAN_WARPS) * STAGES * BYTES;
  static constexpr int AHEAD = STAGES - 1;        // segments under way before the first is waited for
  static constexpr int V = 16 / static_cast<int>(sizeof(T)), UNITS = CH / V, EACH = 32 / UNITS;       // units of a row, rows a warp copies at once
  static_assert(FEED != BY_UNITS || N % EACH == 0, "a copy stays in its segment");
  char* base;
  int fill, read;                                 // bytes from the base: the stage to be filled, to be read
  int mine;                                       // this lane's elements of a row
  int begin[PIECES ? ARRAYS : 1], step[PIECES ? ARRAYS : 1];      // bytes: where a segment's first row begins in a piece, from row to row

  __device__ __forceinline__ Ring(char* shared, int warp, int lane) : base(shared + static_cast<size_t>(warp) * STAGES * BYTES), fill(0), read(0) {
    mine = lane / (CH / 2) * NEXT_SEG + lane % (CH / 2) * static_cast<int>(sizeof(T)) * (FEED == BY_ELEMENTS ? 1 : 2);
  }
  // Says where a matrix's segments lie: p is the first element of one of them; it is the same for every tile's.
  __device__ __forceinline__ void lies(int array, const T* p, long long ld) {
    if constexpr (PIECES) {
      begin[array] = uniform(static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15));
      step[array] = static_cast<int>(ld * static_cast<long long>(sizeof(T)) & 15);
    }
  }
  __device__ __forceinline__ int at(int array, int row) const {
    if constexpr (PIECES) return mine + ((begin[array] + row % V * step[array]) & 15);
    return mine;
  }

  // This lane's first element of a segment that begins at p; in pieces, the segment's.
  template <typename P>
  static __device__ __forceinline__ P* own(P* p, long long ld) {
    const int lane = threadIdx.x & 31;
    if constexpr (FEED == BY_UNITS) return p + lane / UNITS * ld + lane % UNITS * V;
    else return p;
  }
  static __device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  }
  // Rows from own(); `channels` remain from the slice's first.  first, last: the matrix's.
  __device__ __forceinline__ void copy(int array, const T* from, long long ld, int rows, int channels, const T* first, const T* last) {
    const int lane = threadIdx.x & 31;
    const uint32_t area = twa_smem_u32(base + fill + array * AREA);
    if constexpr (FEED == BY_UNITS) {
      const int upto = lane % UNITS * V < channels ? rows - lane / UNITS : 0;
#pragma unroll
      for (int i = 0; i < SEGS * N; i += EACH) {
        if (i < upto) copy_async(area + lane * 16 + i / N * NEXT_SEG + i % N * ROW, from);
        from += EACH * ld;
      }
    } else {
      constexpr int OF_ROW = ROW / 16, ROWS = 32 / OF_ROW;                                // pieces of a row, rows a warp copies at once
      const int piece = lane % OF_ROW * 16, upto = lane < ROWS * OF_ROW ? rows - lane / OF_ROW : 0;
      const int bytes = min(channels, CH) * static_cast<int>(sizeof(T));
      const uintptr_t lo = reinterpret_cast<uintptr_t>(first), hi = reinterpret_cast<uintptr_t>(last + 1);
      uintptr_t row = reinterpret_cast<uintptr_t>(from);
      const bool edge = row < lo + 16 || row + (rows - 1) * ld * sizeof(T) + CH * sizeof(T) + 16 > hi;       // of the matrix; true of the whole warp
      row += lane / OF_ROW * ld * sizeof(T);
#pragma unroll
      for (int i = 0; i < N; i += ROWS) {
        const uintptr_t p = (row & ~static_cast<uintptr_t>(15)) + piece;
        if (i < upto && piece < bytes + static_cast<int>(row & 15)) {
          if (!edge || (p >= lo && p + 16 <= hi)) {
            copy_async(area + i * ROW + lane * 16, reinterpret_cast<const void*>(p));
          } else {                                 // reaches out of the matrix: what lies in it, by the element
            for (int e = 0; e < 16; e += sizeof(T))
              if (p + e >= lo && p + e < hi)
                *reinterpret_cast<T*>(base + fill + array * AREA + i * ROW + lane * 16 + e) = *reinterpret_cast<const T*>(p + e);
          }
        }
        row += ROWS * ld * sizeof(T);
      }
    }
  }
  // Ends the copies of one segment.
  __device__ __forceinline__ void filled() {
    asm volatile("cp.async.commit_group;" ::: "memory");
    fill = fill == (STAGES - 1) * BYTES ? 0 : fill + BYTES;
  }
  // Waits for the oldest segment.
  __device__ __forceinline__ void wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
    __syncwarp();
    if constexpr (PIECES) {                        // rows' places are found anew for every segment: they would fill the registers
#pragma unroll
      for (int i = 0; i < ARRAYS; ++i) asm volatile("" : "+r"(begin[i]));
    }
  }
  __device__ __forceinline__ Pair<T> get(int array, int row) const {
    const char* p = base + read + array * AREA + row * ROW + at(array, row);
    Pair<T> v;
    if constexpr (FEED == BY_ELEMENTS && sizeof(T) == 2) v.r = *reinterpret_cast<const unsigned short*>(p) | static_cast<uint32_t>(*reinterpret_cast<const unsigned short*>(p + 64)) << 16;
    else if constexpr (FEED == BY_ELEMENTS) v.r = make_float2(*reinterpret_cast<const float*>(p), *reinterpret_cast<const float*>(p + 128));
    else v = *reinterpret_cast<const Pair<T>*>(p);
    return v;
  }
  // By units: a result in the place of what get() gave, and the whole segment of them to memory, from own().
  __device__ __forceinline__ void put(int array, int row, float lo, float hi) const {
    Pair<T>::template store<true>(reinterpret_cast<T*>(base + read + array * AREA + row * ROW + mine), lo, hi, 2);
  }
  __device__ __forceinline__ void flush(int array, T* to, long long ld, int channels) const {
    const int lane = threadIdx.x & 31;
    const char* from = base + read + array * AREA + lane * 16;
    if (lane % UNITS * V >= channels) return;
#pragma unroll
    for (int i = 0; i < SEGS * N; i += EACH) {
      *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from + i / N * NEXT_SEG + i % N * ROW);
      to += EACH * ld;
    }
  }
  __device__ __forceinline__ void done() {
    read = read == (STAGES - 1) * BYTES ? 0 : read + BYTES;
    __syncwarp();                                 // other lanes fill this stage again
  }
};

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
// next ones go beside those being read, or, where the ring leaves no room, the segments' once and a barrier behind the reading.
template <int PAIRS, int SETS>
struct Joins {
  Map seg[SETS][SCAN_WARPS][PAIRS];
  twa_f2 carry[2][PAIRS];
};
// The same of the tiles of a cluster's blocks, and how they arrive.  stop: what a block does in the round after: GO_ON, STOP, or, 1 + w,
// let its warp w take its wait for one that ran out.
enum { STOP = -1, GO_ON = 0 };
template <int PAIRS>
struct Tiles {
  Map tile[2][MAX_CLUSTER][PAIRS];
  unsigned long long arrived[2];
  int abort_flag;
  int stop[2];
  static constexpr unsigned BYTES = PAIRS * sizeof(Map);         // of one block's
};

// The blocks of a cluster tell each other what their tiles make of a state: every warp joins its block's segments' maps, from the
// first on (FORWARD) or from the last, and the warp of each rank sends the tile's to that block, whose barrier counts the bytes.
// (A barrier of the whole cluster instead would also wait until every thread's results are in memory: 1 x 65536 x 512 float32
// both directions 277 us, so 237.)  Two sets take turns: a block sends into one again only after it has the maps of the
// round between, which the receiver sends when all its warps have read the first.
// A barrier is told what to wait for next as soon as it has been waited for, not when that round's maps are due.
// Warps wait each for themselves.  One to which the maps do not come in time reports it, even where another of its block has had them
// just before the limit, and tells its block to stop, which from the next round on sends nothing, waits for nothing and stores nothing:
// its maps would be wrong, and others would take those of later rounds for missing ones.  So every map that arrives is right, and every
// row that is stored.  False: the maps are not here.
template <bool FORWARD, int FEED, int CH, int SETS>
__device__ __forceinline__ bool share_tile(const ScanArgs& a, const Joins<CH / 2, SETS>& joins, Tiles<CH / 2>& tiles, const Place<FEED, CH>& at, int turn,
                                           unsigned& phases, int seq) {
  const int stop = tiles.stop[turn ^ 1];           // written before the barrier that the block has passed
  if (at.warp < at.ranks) {
    Map all = joins.seg[turn % SETS][FORWARD ? 0 : SCAN_WARPS - 1][at.pair];
#pragma unroll
    for (int i = 1; i < SCAN_WARPS; ++i) all = joins.seg[turn % SETS][FORWARD ? i : SCAN_WARPS - 1 - i][at.pair].after(all);
    if (at.seg == 0 && stop != STOP) {
      uint32_t to, bar;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(twa_smem_u32(&tiles.tile[turn][at.rank][at.pair])), "r"(at.warp));
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(twa_smem_u32(&tiles.arrived[turn])), "r"(at.warp));
      asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(to), "l"(all.A), "l"(all.B), "r"(bar)
                   : "memory");
    }
  }
  const bool good = stop != STOP && stop != 1 + at.warp && twa_wait(&tiles.arrived[turn], phases >> turn & 1, &tiles.abort_flag, a.wait_limit_ns);
  phases ^= 1u << turn;
  if (__all_sync(0xffffffffu, good)) {             // a warp goes on as one
    if (threadIdx.x == 0) twa_mbar_expect_tx(twa_smem_u32(&tiles.arrived[turn]), at.ranks * Tiles<CH / 2>::BYTES);
    return true;
  }
  if (at.lane == 0) {
    tiles.stop[turn] = STOP;
    twa_set_status(a.status, TWA_ERR_TIMEOUT, seq);
  }
  __syncwarp();
  return false;
}
static_assert(MAX_CLUSTER <= SCAN_WARPS, "a warp for every rank");
// Whether a warp's block was told to stop, by the warp itself or, a round ago, by another: what it has of a state is not the sequence's.
template <int PAIRS>
__device__ __forceinline__ bool scan_stopped(const Tiles<PAIRS>& tiles, int ranks) {
  return ranks > 1 && (tiles.stop[0] == STOP || tiles.stop[1] == STOP);
}

// The sequence that has `place` longer ones before it, of at most SCAN_THREADS; by the whole block, which has `shared` for it.
__device__ __forceinline__ int by_length(const ScanArgs& a, int place, int* shared) {
  const int own = threadIdx.x;
  const int len = own < a.sequences ? scan_span<true>(a, own, false).len : -1;
  shared[own] = len;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < a.sequences; ++i) before += shared[i] > len || (shared[i] == len && i < own) ? 1 : 0;
  __syncthreads();
  if (own < a.sequences && before == place) shared[0] = own;
  __syncthreads();
  const int seq = shared[0];
  __syncthreads();
  return seq;
}

// GROUP sequences of a slice of channels a block.  The ones of at most SEG rows go to one warp each, the others to the block, or
// the cluster.  The state that leaves a sequence may lie where the one that enters it does, which every block of a cluster reads: it is
// written behind the barrier at the end.  Offsets on the device are read once and handed on: a block, and a cluster, has one opinion of where its sequences lie.
// (Equal lengths are a matter of their own: what follows from them alone stays in uniform registers; 8 x 2048 x 2048 bfloat16 forward
// 47 us, 53 when they come the same way.)
template <typename Direction, int GROUP, bool RAGGED>
__device__ __forceinline__ void scan_block(const ScanArgs& a) {
  typedef Tiles<Direction::CHANNELS / 2> T;
  extern __shared__ __align__(16) char shared[];
  __shared__ Joins<Direction::CHANNELS / 2, Direction::SETS> joins;
  T& tiles = *reinterpret_cast<T*>(shared + Direction::Rows::BLOCK_BYTES);       // of clusters only
  const unsigned task = blockIdx.x / a.cluster;
  const int slice = task % a.slices, first = task / a.slices * GROUP;
  Direction d(a, slice);
  if (a.cluster > 1) {
    if (threadIdx.x == 0) {
      for (int i = 0; i < 2; ++i) twa_mbar_init(twa_smem_u32(&tiles.arrived[i]), 1);
      tiles.abort_flag = 0;
      tiles.stop[0] = GO_ON;
      tiles.stop[1] = a.give_up && (a.give_up - 1) / SCAN_WARPS == d.at.rank ? 1 + (a.give_up - 1) % SCAN_WARPS : GO_ON;
      twa_fence_barrier_init();
      for (int i = 0; i < 2; ++i) twa_mbar_expect_tx(twa_smem_u32(&tiles.arrived[i]), a.cluster * T::BYTES);
    }
    twa_cluster_sync();                            // no block stores into one that has not begun
  }
  int turn = 0, seq = first;
  bool leaves = false;
  twa_f2 state = 0;
  if constexpr (!RAGGED) {
    const Span s = scan_span<false>(a, first, false);
    leaves = d.whole(s, first, shared, joins, tiles, turn, state);
  } else {
    __shared__ unsigned long long begins[GROUP], lengths[GROUP];    // lengths: and the sequence's number above them
    if (d.at.rank == 0) {
      const int from = GROUP == 1 && a.by_length ? by_length(a, first, reinterpret_cast<int*>(shared)) : first;
      if (threadIdx.x < GROUP) {
        const int seq = from + threadIdx.x;
        Span s = {0, -1};
        if (seq < a.sequences) s = scan_span<true>(a, seq, slice == 0);
        const unsigned long long length = static_cast<unsigned long long>(seq) << 32 | static_cast<unsigned>(s.len);
        begins[threadIdx.x] = static_cast<unsigned long long>(s.begin);
        lengths[threadIdx.x] = length;
        for (int r = 1; r < a.cluster; ++r) {
          twa_store_remote(begins + threadIdx.x, r, static_cast<unsigned long long>(s.begin));
          twa_store_remote(lengths + threadIdx.x, r, length);
        }
      }
    }
    if (a.cluster > 1) twa_cluster_sync();
    else __syncthreads();
    auto span = [&](int g) {
      const unsigned lo = uniform(static_cast<int>(begins[g])), hi = uniform(static_cast<int>(begins[g] >> 32));
      return Span{static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo), uniform(static_cast<int>(lengths[g]))};
    };
    auto number = [&](int g) { return uniform(static_cast<int>(lengths[g] >> 32)); };
    if constexpr (GROUP > 1) {
      const Span s = span(d.at.warp);
      if (s.len >= 0 && s.len <= Direction::N) Direction::brief(a, d.at, s, number(d.at.warp));
    }
    for (int g = 0; g < GROUP; ++g) {
      const Span s = span(g);
      if (s.len > Direction::N || (GROUP == 1 && s.len >= 0)) {
        seq = number(g);
        leaves = d.whole(s, seq, shared, joins, tiles, turn, state);
        if (GROUP > 1 && leaves) d.carry(seq, state);              // never in a cluster
      }
    }
  }
  if (a.cluster > 1) twa_cluster_sync();           // none ends while another may still send to it, one whose wait ran out included
  if (GROUP == 1 && leaves) d.carry(seq, state);
}

template <typename Direction, int GROUP, bool RAGGED>
__global__ void __launch_bounds__(SCAN_THREADS, 2) scan_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.dh, a.starts, a.h0, a.states, a.d_last);
  scan_block<Direction, GROUP, RAGGED>(a);
}
// Where no sequence is longer than SEG rows: a warp for each, of each slice.
template <typename Direction>
__global__ void __launch_bounds__(SCAN_THREADS) scan_brief_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.dh, a.h0, a.states, a.d_last);
  const int slice = blockIdx.x % a.slices, seq = blockIdx.x / a.slices * SHORT_GROUP + (threadIdx.x >> 5);
  if (seq < a.sequences) Direction::brief(a, typename Direction::At(a, slice), scan_span<false>(a, seq, false), seq);
}

constexpr int SCAN_RESIDENT = 2;                   // blocks of an SM

// ---- the host's side ------------------------------------------------------------------------------------
// How rows of two pointers and strides can be fetched together.
inline int scan_feed(const void* p, long long ld, size_t size, int channels, int so_far) {
  if (so_far == BY_UNITS && (channels * size % 16 || twa_misaligned_to(p, 16) || ld * size % 16)) so_far = BY_PAIRS;
  if (so_far == BY_PAIRS && (channels % 2 || twa_misaligned_to(p, 2 * size) || ld % 2)) so_far = BY_ELEMENTS;
  return so_far;
}
template <typename Direction, int GROUP, bool RAGGED>
cudaError_t scan_launch(twa_ctx* ctx, const ScanArgs& a) {
  auto kernel = scan_kernel<Direction, GROUP, RAGGED>;
  const size_t smem = Direction::Rows::BLOCK_BYTES + (a.cluster > 1 ? sizeof(Tiles<Direction::CHANNELS / 2>) : 0);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.sequences, GROUP) * a.slices * a.cluster);
  return twa_launch_clusters(ctx->stream, kernel, blocks, a.cluster, SCAN_THREADS, smem, a);
}
template <typename Direction>
cudaError_t scan_launch(twa_ctx* ctx, const ScanArgs& a) {
  return a.starts ? scan_launch<Direction, 1, true>(ctx, a) : scan_launch<Direction, 1, false>(ctx, a);
}
template <template <typename, int, int> class Direction, typename T>
cudaError_t scan_launch(twa_ctx* ctx, ScanArgs& a, int feed) {
  a.cluster = 1;
  // A warp a sequence: all of them where they are short enough, or, of ragged ones, those that are, where most must be.
  const bool short_all = !a.starts && a.tokens <= static_cast<long long>(SEG<T>) * a.sequences;
  if (short_all || (a.starts && 2 * a.tokens <= static_cast<long long>(SEG<T>) * a.sequences)) {
    a.slices = static_cast<int>(twa_ceil_div(a.channels, SCAN_CHANNELS));
    if (short_all) {
      const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.sequences, SHORT_GROUP) * a.slices);
      auto launch = [&](auto kernel) { return twa_launch(ctx->stream, kernel, blocks, SCAN_THREADS, 0, a); };
      return feed == BY_ELEMENTS ? launch(scan_brief_kernel<Direction<T, BY_ELEMENTS, SCAN_CHANNELS>>)
                                 : launch(scan_brief_kernel<Direction<T, BY_PAIRS, SCAN_CHANNELS>>);
    }
    return feed == BY_UNITS   ? scan_launch<Direction<T, BY_UNITS, SCAN_CHANNELS>, SHORT_GROUP, true>(ctx, a)
           : feed == BY_PAIRS ? scan_launch<Direction<T, BY_PAIRS, SCAN_CHANNELS>, SHORT_GROUP, true>(ctx, a)
                              : scan_launch<Direction<T, BY_ELEMENTS, SCAN_CHANNELS>, SHORT_GROUP, true>(ctx, a);
  }
  int channels = SCAN_CHANNELS;
  auto blocks = [&]() { return twa_ceil_div(a.channels, channels) * a.sequences * a.cluster; };
  auto rows = [&]() { return a.cluster * SCAN_WARPS * SEG<T> * (SCAN_CHANNELS / channels); };       // of a round
  // Twice as many where there is room for them and rows enough; ragged sequences wait for the longest, which takes the more blocks
  // (15 ragged sequences of 13138 x 1016 bfloat16, both directions 133 us with one block each, 110 with two).
  const int slots = SCAN_RESIDENT * ctx->sm_count, places = (a.starts ? 2 : 1) * slots;
  auto more = [&]() { return 2 * blocks() <= places && a.tokens > 2LL * rows() * a.sequences; };
  if (ctx->tune_scan_channels && feed == BY_UNITS) channels = ctx->tune_scan_channels;
  else if (feed == BY_UNITS && more()) channels = 32;
  while (a.cluster < MAX_CLUSTER && more()) a.cluster *= 2;
  if (!ctx->tune_scan_channels && channels == 32 && more()) channels = 16;
  if (ctx->tune_scan_cluster) a.cluster = ctx->tune_scan_cluster;
  // Ragged sequences that do not all begin at once go by their length, the longest first (12 ragged sequences of 16384 x 2048 bfloat16
  // 88 us forward in their own order, 72 so); where there are many more than begin at once, a late long one is rare, and finding
  // a block's sequence costs each of them (200 of 32768 x 1024: 70 and 104 us).
  a.by_length = a.starts && a.sequences <= SCAN_THREADS && blocks() > slots && blocks() <= 2 * slots;
  a.slices = static_cast<int>(twa_ceil_div(a.channels, channels));
  if (feed == BY_PAIRS) return scan_launch<Direction<T, BY_PAIRS, SCAN_CHANNELS>>(ctx, a);
  if (feed == BY_ELEMENTS) return scan_launch<Direction<T, BY_ELEMENTS, SCAN_CHANNELS>>(ctx, a);
  return channels == 64   ? scan_launch<Direction<T, BY_UNITS, 64>>(ctx, a)
         : channels == 32 ? scan_launch<Direction<T, BY_UNITS, 32>>(ctx, a)
                          : scan_launch<Direction<T, BY_UNITS, 16>>(ctx, a);
}
template <template <typename, int, int> class Direction>
cudaError_t scan_launch(twa_ctx* ctx, ScanArgs& a, int dtype, int feed) {
  return dtype == TWA_BF16 ? scan_launch<Direction, bf16>(ctx, a, feed) : scan_launch<Direction, float>(ctx, a, feed);
}

// Arguments that both directions have.
inline int scan_check(twa_ctx* ctx, int dtype, int64_t tokens, int channels, const void* starts, int s_type, int sequences) {
  if (!ctx || !twa_dtype_ok(dtype) || tokens < 0 || channels < 1 || sequences < 0 || (starts && !twa_itype_ok(s_type))) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_SCAN_MAX_TOKENS || channels > TWA_SCAN_MAX_CHANNELS || sequences > TWA_SCAN_MAX_SEQUENCES) return TWA_ERR_UNSUPPORTED;
  if (!starts && (sequences ? tokens % sequences : tokens)) return TWA_ERR_INVALID_ARG;
  if (starts && twa_misaligned_to(starts, twa_itype_size(s_type))) return TWA_ERR_MISALIGNED;
  // blocks of a launch
  if (static_cast<long long>(sequences) * twa_ceil_div(channels, SCAN_LEAST_CHANNELS) * MAX_CLUSTER > 0x7FFFFFFFLL) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

}  // namespace
