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
// A lane has two neighbouring channels, a warp a segment of SEG rows of 64 channels, the warps of a block consecutive segments:
// a tile of 64 rows.  Every warp takes its own segment from 0, the segments' (A, L) go through shared memory, and
// every thread joins those before its own with the state that enters the tile.  States are float32.
#pragma once

#include "twa_ops.cuh"

namespace {

constexpr int SCAN_WARPS = 8, SCAN_THREADS = SCAN_WARPS * 32;
constexpr int SEG = 8;                             // rows of a segment
constexpr int SCAN_ROWS = SCAN_WARPS * SEG;        // of a tile, and from one kept state to the next
constexpr int SCAN_CHANNELS = 64;                  // of a block
constexpr int SHORT_GROUP = SCAN_WARPS;            // sequences of a block where most are short
constexpr int MAX_CLUSTER = 8;                     // blocks along a sequence

struct ScanArgs {
  const void *x, *f, *dh;
  void *h, *dx, *df;
  long long ldx, ldf, lddh, ldh, lddx, lddf;
  long long tokens;
  const void* starts;
  int s_type, sequences, channels, slices, cluster;
  const float* h0;
  float* h_last;
  float* states;
  const float* d_last;
  float* dh0;
  int* status;
};

// Rows of a sequence; len -1: its offsets are wrong and it is left alone.
struct Span {
  long long begin, len;
};
__device__ __forceinline__ Span scan_span(const ScanArgs& a, int seq, bool report) {
  if (!a.starts) {
    const long long each = a.tokens / a.sequences;
    return {seq * each, each};
  }
  const long long b = twa_load_id(a.starts, a.s_type, seq), e = twa_load_id(a.starts, a.s_type, seq + 1);
  if (b < 0 || e < b || e > a.tokens) {
    if (report) twa_set_status(a.status, TWA_ERR_INVALID_ARG, seq);
    return {0, -1};
  }
  return {b, e - b};
}
// The first of a sequence's kept states: those of sequences before it end before this place, for
// (b + len) / R + 1 >= b / R + ceil(len / R).
__device__ __forceinline__ long long scan_slot(const Span& s, int seq) { return s.begin / SCAN_ROWS + seq; }

// Two neighbouring elements as they lie in memory.  PACKED: one access, on the pair's boundary; otherwise one each, `n` of them.
template <typename T>
struct Pair;
template <>
struct Pair<float> {
  float2 r;
  template <bool PACKED>
  __device__ __forceinline__ void load(const float* p, int n) {
    if constexpr (PACKED) r = __ldg(reinterpret_cast<const float2*>(p));
    else {
      r.x = __ldg(p);
      r.y = n > 1 ? __ldg(p + 1) : 0.0f;
    }
  }
  __device__ __forceinline__ float lo() const { return r.x; }
  __device__ __forceinline__ float hi() const { return r.y; }
  __device__ __forceinline__ twa_f2 both() const { return twa_pair(r.x, r.y); }
  template <bool PACKED>
  static __device__ __forceinline__ void store(float* p, float a, float b, int n) {
    if constexpr (PACKED) *reinterpret_cast<float2*>(p) = make_float2(a, b);
    else {
      p[0] = a;
      if (n > 1) p[1] = b;
    }
  }
};
template <>
struct Pair<bf16> {
  uint32_t r;
  template <bool PACKED>
  __device__ __forceinline__ void load(const bf16* p, int n) {
    if constexpr (PACKED) r = __ldg(reinterpret_cast<const uint32_t*>(p));
    else {
      const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
      r = __ldg(q);
      if (n > 1) r |= static_cast<uint32_t>(__ldg(q + 1)) << 16;
    }
  }
  __device__ __forceinline__ float lo() const { return twa_bf16_lo(r); }
  __device__ __forceinline__ float hi() const { return twa_bf16_hi(r); }
  __device__ __forceinline__ twa_f2 both() const { return twa_pair(lo(), hi()); }
  template <bool PACKED>
  static __device__ __forceinline__ void store(bf16* p, float a, float b, int n) {
    if constexpr (PACKED) *reinterpret_cast<uint32_t*>(p) = twa_bf16_pair(a, b);
    else {
      p[0] = twa_from_float<bf16>(a);
      if (n > 1) p[1] = twa_from_float<bf16>(b);
    }
  }
};

// -q of two gates; their signs say which form a step takes.  The exponential of a bfloat16 gate may err by some units of float32,
// that of a float32 gate may not.
template <typename T>
__device__ __forceinline__ float scan_exp(float f) {
  return sizeof(T) == 2 ? __expf(f) : expf(f);
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
  twa_unpair(twa_add2(twa_pair(1.0f), twa_pair(scan_exp<T>(fabsf(f.lo())), scan_exp<T>(fabsf(f.hi())))), a, b);
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
__device__ __forceinline__ twa_f2 scan_step(twa_f2 n, twa_f2 h, twa_f2 x) { return twa_fma2(n, scan_minus(h, x), scan_pick(n, h, x)); }
// a times v: what a step makes of a state where x is 0.
__device__ __forceinline__ twa_f2 scan_decay(twa_f2 n, twa_f2 v) { return twa_fma2(n, v, scan_pick(n, v, twa_pair(0.0f))); }

// ---- rows on their way --------------------------------------------------------------------------------
// How a warp fetches its segments' rows: in units of 16 bytes, any lane's; in pairs, each lane its own; or element by element.
enum { BY_UNITS, BY_PAIRS, BY_ELEMENTS };

// A ring of a warp's segments in shared memory, STAGES deep, of ARRAYS matrices.  The copies are asynchronous but for those by
// elements, which go through registers one segment ahead.
template <typename T, int FEED, int ARRAYS, int STAGES>
struct Ring {
  static constexpr int ROW = SCAN_CHANNELS * sizeof(T), BYTES = ARRAYS * SEG * ROW;     // of a row, of a segment
  static constexpr size_t BLOCK_BYTES = static_cast<size_t>(SCAN_WARPS) * STAGES * BYTES;
  char* base;
  Pair<T> held[FEED == BY_ELEMENTS ? ARRAYS * SEG : 1];
  int fill, read;

  __device__ __forceinline__ Ring(char* shared, int warp) : base(shared + static_cast<size_t>(warp) * STAGES * BYTES), fill(0), read(0) {}

  __device__ __forceinline__ void copy(int array, const T* p, long long ld, int rows, int channels) {
    const int lane = threadIdx.x & 31;
    if constexpr (FEED == BY_UNITS) {
      constexpr int UNITS = ROW / 16, EACH = 32 / UNITS;
      const int u = lane % UNITS, r0 = lane / UNITS;
      const uint32_t to = twa_smem_u32(base + fill * BYTES + array * SEG * ROW + r0 * ROW + u * 16);
      const T* from = p + r0 * ld + u * (16 / static_cast<int>(sizeof(T)));
      const bool in = u * (16 / static_cast<int>(sizeof(T))) < channels;
#pragma unroll
      for (int i = 0; i < SEG / EACH; ++i)
        if (in && r0 + i * EACH < rows)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * EACH * ROW), "l"(from + i * EACH * ld) : "memory");
    } else if constexpr (FEED == BY_PAIRS) {
      const uint32_t to = twa_smem_u32(base + fill * BYTES + array * SEG * ROW + lane * 2 * sizeof(T));
      const T* from = p + 2 * lane;
#pragma unroll
      for (int i = 0; i < SEG; ++i)
        if (2 * lane < channels && i < rows)
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to + i * ROW), "l"(from + i * ld), "n"(2 * sizeof(T)) : "memory");
    } else {
      const T* from = p + 2 * lane;
#pragma unroll
      for (int i = 0; i < SEG; ++i)
        if (2 * lane < channels && i < rows) held[array * SEG + i].template load<false>(from + i * ld, channels - 2 * lane);
    }
  }
  // Ends the copies of one segment.
  __device__ __forceinline__ void filled() {
    if constexpr (FEED != BY_ELEMENTS) asm volatile("cp.async.commit_group;" ::: "memory");
    fill = fill + 1 == STAGES ? 0 : fill + 1;
  }
  // Waits for the oldest segment.
  __device__ __forceinline__ void wait() {
    if constexpr (FEED == BY_ELEMENTS) {
      const int lane = threadIdx.x & 31;
#pragma unroll
      for (int i = 0; i < ARRAYS * SEG; ++i) *reinterpret_cast<Pair<T>*>(base + i * ROW + lane * 2 * sizeof(T)) = held[i];
    } else {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      if (FEED == BY_UNITS) __syncwarp();
    }
  }
  __device__ __forceinline__ Pair<T> get(int array, int row) const {
    const int stage = FEED == BY_ELEMENTS ? 0 : read;
    return *reinterpret_cast<const Pair<T>*>(base + stage * BYTES + (array * SEG + row) * ROW + (threadIdx.x & 31) * 2 * sizeof(T));
  }
  __device__ __forceinline__ void done() {
    read = read + 1 == STAGES ? 0 : read + 1;
    if (FEED == BY_UNITS) __syncwarp();           // other lanes fill this stage again
  }
  // Segments that are under way before the first one is waited for.
  static constexpr int AHEAD = FEED == BY_ELEMENTS ? 1 : STAGES - 1;
};

// Two neighbouring channels of a row of float32 states.
__device__ __forceinline__ twa_f2 scan_state(const float* p, long long row, int channels, int c, int n) {
  if (!p) return 0;
  return twa_pair(n > 0 ? p[row * channels + c] : 0.0f, n > 1 ? p[row * channels + c + 1] : 0.0f);
}
__device__ __forceinline__ void scan_keep(float* p, long long row, int channels, int c, int n, twa_f2 v) {
  if (!p) return;
  float lo, hi;
  twa_unpair(v, lo, hi);
  if (n > 0) p[row * channels + c] = lo;
  if (n > 1) p[row * channels + c + 1] = hi;
}

}  // namespace
