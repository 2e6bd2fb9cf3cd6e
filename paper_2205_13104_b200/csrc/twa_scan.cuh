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

struct ScanArgs {
  const void *x, *f, *dh;
  void *h, *dx, *df;
  long long ldx, ldf, lddh, ldh, lddx, lddf;
  long long tokens;
  const void* starts;
  int s_type, sequences, channels, slices;
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
template <typename T, bool PACKED>
struct Pair;
template <bool PACKED>
struct Pair<float, PACKED> {
  float2 r;
  __device__ __forceinline__ void load(const float* p, int n) {
    if constexpr (PACKED) r = __ldg(reinterpret_cast<const float2*>(p));
    else {
      r.x = __ldg(p);
      r.y = n > 1 ? __ldg(p + 1) : 0.0f;
    }
  }
  __device__ __forceinline__ float get(int c) const { return c ? r.y : r.x; }
  static __device__ __forceinline__ void store(float* p, float a, float b, int n) {
    if constexpr (PACKED) *reinterpret_cast<float2*>(p) = make_float2(a, b);
    else {
      p[0] = a;
      if (n > 1) p[1] = b;
    }
  }
};
template <bool PACKED>
struct Pair<bf16, PACKED> {
  uint32_t r;
  __device__ __forceinline__ void load(const bf16* p, int n) {
    if constexpr (PACKED) r = __ldg(reinterpret_cast<const uint32_t*>(p));
    else {
      const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
      r = __ldg(q);
      if (n > 1) r |= static_cast<uint32_t>(__ldg(q + 1)) << 16;
    }
  }
  __device__ __forceinline__ float get(int c) const { return c ? twa_bf16_hi(r) : twa_bf16_lo(r); }
  static __device__ __forceinline__ void store(bf16* p, float a, float b, int n) {
    if constexpr (PACKED) *reinterpret_cast<uint32_t*>(p) = twa_bf16_pair(a, b);
    else {
      p[0] = twa_from_float<bf16>(a);
      if (n > 1) p[1] = twa_from_float<bf16>(b);
    }
  }
};

// q of a gate.  The exponential of a bfloat16 gate may err by some units of float32, that of a float32 gate may not.
template <typename T>
__device__ __forceinline__ float scan_gate(float f) {
  const float e = sizeof(T) == 2 ? __expf(fabsf(f)) : expf(fabsf(f));
  return copysignf(__frcp_rn(1.0f + e), f);
}
__device__ __forceinline__ bool scan_open(float q) { return __float_as_int(q) >= 0; }
__device__ __forceinline__ float scan_step(float q, float h, float x) { return fmaf(q, x - h, scan_open(q) ? h : x); }
// a times v: what a step makes of a state where x is 0.
__device__ __forceinline__ float scan_decay(float q, float v) { return fmaf(-q, v, scan_open(q) ? v : 0.0f); }

// Two neighbouring channels of a row of float32 states.
__device__ __forceinline__ void scan_state(const float* p, long long row, int channels, int c, int n, float* v) {
  v[0] = v[1] = 0.0f;
  if (!p) return;
  if (n > 0) v[0] = p[row * channels + c];
  if (n > 1) v[1] = p[row * channels + c + 1];
}
__device__ __forceinline__ void scan_keep(float* p, long long row, int channels, int c, int n, const float* v) {
  if (!p) return;
  if (n > 0) p[row * channels + c] = v[0];
  if (n > 1) p[row * channels + c + 1] = v[1];
}

}  // namespace
