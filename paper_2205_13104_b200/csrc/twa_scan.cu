// Gated linear recurrence, both directions; the forms that are used here stand in twa_scan.cuh.
//
//   forward    h_t = a_t h_{t-1} + (1 - a_t) x_t,   a_t = sigmoid(f_t)
//   backward   G_t = dh_t + a_{t+1} G_{t+1},   dx_t = (1 - a_t) G_t,   df_t = a_t (1 - a_t) (h_{t-1} - x_t) G_t
//
// Backward the states before every row are taken again from those that the forward pass kept in float32, one every 64 rows, and
// what goes from row to row is k_t = a_t G_t, affine in the one that enters: k = A k_in + M with the same A as forward.
#include "twa_scan.cuh"

namespace {

template <typename T, bool PACKED>
struct ScanForward {
  const ScanArgs& a;
  const int lane, warp, c, n;                      // channels c, c + 1; n of them exist
  Pair<T, PACKED> rx[SEG], rf[SEG];
  float A[SEG][2], L[SEG][2];                      // of the rows up to each

  __device__ __forceinline__ ScanForward(const ScanArgs& args, int slice)
      : a(args), lane(threadIdx.x & 31), warp(threadIdx.x >> 5), c(slice * SCAN_CHANNELS + 2 * (threadIdx.x & 31)),
        n(args.channels - c < 2 ? (args.channels - c < 0 ? 0 : args.channels - c) : 2) {}

  __device__ __forceinline__ void load(long long row, int rows) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx + c;
    const T* f = static_cast<const T*>(a.f) + row * a.ldf + c;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows && n > 0) {
        rx[i].load(x + i * a.ldx, n);
        rf[i].load(f + i * a.ldf, n);
      }
  }
  // A and L of the rows; returns those of the segment.
  __device__ __forceinline__ float4 local(int rows) {
    float s[2] = {1.0f, 1.0f}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float q = scan_gate<T>(rf[i].get(e));
          s[e] = scan_decay(q, s[e]);
          l[e] = scan_step(q, l[e], rx[i].get(e));
          A[i][e] = s[e];
          L[i][e] = l[e];
        }
      }
    return make_float4(s[0], l[0], s[1], l[1]);
  }
  __device__ __forceinline__ void store(long long row, int rows, const float* in) {
    T* h = static_cast<T*>(a.h) + row * a.ldh + c;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows && n > 0)
        Pair<T, PACKED>::store(h + i * a.ldh, fmaf(A[i][0], in[0], L[i][0]), fmaf(A[i][1], in[1], L[i][1]), n);
  }

  // A sequence of at most SEG rows, by one warp.
  __device__ __forceinline__ void brief(const Span& s, int seq) {
    float state[2];
    load(s.begin, static_cast<int>(s.len));
    scan_state(a.h0, seq, a.channels, c, n, state);
    if (s.len) scan_keep(a.states, scan_slot(s, seq), a.channels, c, n, state);
    const float4 end = local(static_cast<int>(s.len));
    store(s.begin, static_cast<int>(s.len), state);
    const float last[2] = {fmaf(end.x, state[0], end.y), fmaf(end.z, state[1], end.w)};
    scan_keep(a.h_last, seq, a.channels, c, n, last);
  }

  // A sequence by the whole block.
  __device__ __forceinline__ void whole(const Span& s, int seq, float4 (*seg)[SCAN_WARPS][32], int& turn) {
    float state[2];
    scan_state(a.h0, seq, a.channels, c, n, state);
    long long slot = scan_slot(s, seq);
    for (long long t = 0; t < s.len; t += SCAN_ROWS, ++slot) {
      const long long mine = t + warp * SEG;
      const int rows = static_cast<int>(s.len - mine < SEG ? (s.len - mine < 0 ? 0 : s.len - mine) : SEG);
      load(s.begin + mine, rows);
      if (warp == 0) scan_keep(a.states, slot, a.channels, c, n, state);
      seg[turn][warp][lane] = local(rows);
      __syncthreads();
      float in[2];
#pragma unroll
      for (int w = 0; w < SCAN_WARPS; ++w) {
        if (w == warp) in[0] = state[0], in[1] = state[1];
        const float4 m = seg[turn][w][lane];
        state[0] = fmaf(m.x, state[0], m.y);
        state[1] = fmaf(m.z, state[1], m.w);
      }
      turn ^= 1;                                   // the next tile's segments go beside those that are being read
      store(s.begin + mine, rows, in);
    }
    if (warp == 0) scan_keep(a.h_last, seq, a.channels, c, n, state);
  }
};

template <typename T, bool PACKED>
struct ScanBackward {
  const ScanArgs& a;
  const int lane, warp, c, n;
  Pair<T, PACKED> rx[SEG], rf[SEG], rd[SEG];
  float q[SEG][2], d[SEG][2];                      // d: h_{t-1} - x_t

  __device__ __forceinline__ ScanBackward(const ScanArgs& args, int slice)
      : a(args), lane(threadIdx.x & 31), warp(threadIdx.x >> 5), c(slice * SCAN_CHANNELS + 2 * (threadIdx.x & 31)),
        n(args.channels - c < 2 ? (args.channels - c < 0 ? 0 : args.channels - c) : 2) {}

  __device__ __forceinline__ void load(long long row, int rows) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx + c;
    const T* f = static_cast<const T*>(a.f) + row * a.ldf + c;
    const T* g = static_cast<const T*>(a.dh) + row * a.lddh + c;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows && n > 0) {
        rx[i].load(x + i * a.ldx, n);
        rf[i].load(f + i * a.ldf, n);
        rd[i].load(g + i * a.lddh, n);
      }
  }
  // The gates; A, L and M of the segment.
  __device__ __forceinline__ void local(int rows, float* A, float* L, float* M) {
#pragma unroll
    for (int e = 0; e < 2; ++e) A[e] = 1.0f, L[e] = M[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          q[i][e] = scan_gate<T>(rf[i].get(e));
          A[e] = scan_decay(q[i][e], A[e]);
          L[e] = scan_step(q[i][e], L[e], rx[i].get(e));
        }
      }
#pragma unroll
    for (int i = SEG - 1; i >= 0; --i)
      if (i < rows) {
#pragma unroll
        for (int e = 0; e < 2; ++e) M[e] = scan_decay(q[i][e], rd[i].get(e) + M[e]);
      }
  }
  // Gradients of the rows from the state h before the first of them and k from behind the last one, which becomes that of the first.
  __device__ __forceinline__ void store(long long row, int rows, float* h, float* k) {
    T* dx = static_cast<T*>(a.dx) + row * a.lddx + c;
    T* df = static_cast<T*>(a.df) + row * a.lddf + c;
#pragma unroll
    for (int i = 0; i < SEG; ++i)
      if (i < rows) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = rx[i].get(e);
          d[i][e] = h[e] - x;
          h[e] = scan_step(q[i][e], h[e], x);
        }
      }
#pragma unroll
    for (int i = SEG - 1; i >= 0; --i)
      if (i < rows) {
        float gx[2], gf[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float g = rd[i].get(e) + k[e], s = fabsf(q[i][e]);
          gx[e] = fmaf(q[i][e], g, scan_open(q[i][e]) ? 0.0f : g);       // (1 - a) g
          gf[e] = fmaf(-s, s, s) * d[i][e] * g;
          k[e] = scan_decay(q[i][e], g);
        }
        if (n > 0) {
          Pair<T, PACKED>::store(dx + i * a.lddx, gx[0], gx[1], n);
          Pair<T, PACKED>::store(df + i * a.lddf, gf[0], gf[1], n);
        }
      }
  }

  __device__ __forceinline__ void brief(const Span& s, int seq) {
    float h[2] = {0.0f, 0.0f}, k[2], A[2], L[2], M[2];
    const int rows = static_cast<int>(s.len);
    load(s.begin, rows);
    if (rows) scan_state(a.states, scan_slot(s, seq), a.channels, c, n, h);
    scan_state(a.d_last, seq, a.channels, c, n, k);
    local(rows, A, L, M);
    store(s.begin, rows, h, k);
    scan_keep(a.dh0, seq, a.channels, c, n, k);
  }

  __device__ __forceinline__ void whole(const Span& s, int seq, float2 (*seg)[SCAN_WARPS][3][32], int& turn) {
    float k[2];
    scan_state(a.d_last, seq, a.channels, c, n, k);
    const long long tiles = (s.len + SCAN_ROWS - 1) / SCAN_ROWS;
    for (long long tile = tiles - 1; tile >= 0; --tile) {
      const long long mine = tile * SCAN_ROWS + warp * SEG;
      const int rows = static_cast<int>(s.len - mine < SEG ? (s.len - mine < 0 ? 0 : s.len - mine) : SEG);
      float h[2], A[2], L[2], M[2], in[2];
      load(s.begin + mine, rows);
      scan_state(a.states, scan_slot(s, seq) + tile, a.channels, c, n, h);
      local(rows, A, L, M);
      seg[turn][warp][0][lane] = make_float2(A[0], A[1]);
      seg[turn][warp][1][lane] = make_float2(L[0], L[1]);
      seg[turn][warp][2][lane] = make_float2(M[0], M[1]);
      __syncthreads();
#pragma unroll
      for (int w = 0; w < SCAN_WARPS; ++w)
        if (w < warp) {
          const float2 mA = seg[turn][w][0][lane], mL = seg[turn][w][1][lane];
          h[0] = fmaf(mA.x, h[0], mL.x);
          h[1] = fmaf(mA.y, h[1], mL.y);
        }
#pragma unroll
      for (int w = SCAN_WARPS - 1; w >= 0; --w) {
        if (w == warp) in[0] = k[0], in[1] = k[1];
        const float2 mA = seg[turn][w][0][lane], mM = seg[turn][w][2][lane];
        k[0] = fmaf(mA.x, k[0], mM.x);
        k[1] = fmaf(mA.y, k[1], mM.y);
      }
      turn ^= 1;
      store(s.begin + mine, rows, h, in);
    }
    if (warp == 0) scan_keep(a.dh0, seq, a.channels, c, n, k);
  }
};

// GROUP sequences of a slice of channels a block.  The ones of at most SEG rows go to one warp each, the others to the block.
template <typename Direction, typename Shared, int GROUP>
__device__ __forceinline__ void scan_block(const ScanArgs& a, Shared shared) {
  const int slice = blockIdx.x % a.slices, first = blockIdx.x / a.slices * GROUP;
  Direction d(a, slice);
  if (GROUP > 1) {
    const int seq = first + d.warp;
    if (seq < a.sequences) {
      const Span s = scan_span(a, seq, slice == 0 && d.lane == 0);
      if (s.len >= 0 && s.len <= SEG) d.brief(s, seq);
    }
  }
  int turn = 0;
  for (int g = 0; g < GROUP; ++g) {
    const int seq = first + g;
    if (seq >= a.sequences) break;
    const Span s = scan_span(a, seq, GROUP == 1 && slice == 0 && threadIdx.x == 0);
    if (s.len > SEG || (GROUP == 1 && s.len >= 0)) d.whole(s, seq, shared, turn);
  }
}

template <typename T, bool PACKED, int GROUP>
__global__ void __launch_bounds__(SCAN_THREADS) scan_forward_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.starts, a.h0);
  __shared__ float4 seg[2][SCAN_WARPS][32];
  scan_block<ScanForward<T, PACKED>, float4(*)[SCAN_WARPS][32], GROUP>(a, seg);
}
template <typename T, bool PACKED, int GROUP>
__global__ void __launch_bounds__(SCAN_THREADS) scan_backward_kernel(ScanArgs a) {
  twa_begin(a.x, a.f, a.dh, a.starts, a.states, a.d_last);
  __shared__ float2 seg[2][SCAN_WARPS][3][32];
  scan_block<ScanBackward<T, PACKED>, float2(*)[SCAN_WARPS][3][32], GROUP>(a, seg);
}

bool scan_packs(const void* p, long long ld, size_t size) { return !twa_misaligned_to(p, 2 * size) && ld % 2 == 0; }

template <typename T>
void scan_launch(twa_ctx* ctx, const ScanArgs& a, bool back, bool packs, bool brief) {
  const unsigned blocks = static_cast<unsigned>(twa_ceil_div(a.sequences, brief ? SHORT_GROUP : 1) * a.slices);
  auto launch = [&](auto kernel) { twa_launch(ctx->stream, kernel, blocks, SCAN_THREADS, 0, a); };
  if (back) {
    if (packs) brief ? launch(scan_backward_kernel<T, true, SHORT_GROUP>) : launch(scan_backward_kernel<T, true, 1>);
    else brief ? launch(scan_backward_kernel<T, false, SHORT_GROUP>) : launch(scan_backward_kernel<T, false, 1>);
  } else {
    if (packs) brief ? launch(scan_forward_kernel<T, true, SHORT_GROUP>) : launch(scan_forward_kernel<T, true, 1>);
    else brief ? launch(scan_forward_kernel<T, false, SHORT_GROUP>) : launch(scan_forward_kernel<T, false, 1>);
  }
}

// Arguments that both directions have.
int scan_check(twa_ctx* ctx, int dtype, int64_t tokens, int channels, const void* starts, int s_type, int sequences) {
  if (!ctx || !twa_dtype_ok(dtype) || tokens < 0 || channels < 1 || sequences < 0 || (starts && !twa_itype_ok(s_type))) return TWA_ERR_INVALID_ARG;
  if (tokens > TWA_SCAN_MAX_TOKENS || channels > TWA_SCAN_MAX_CHANNELS || sequences > TWA_SCAN_MAX_SEQUENCES) return TWA_ERR_UNSUPPORTED;
  if (!starts && (sequences ? tokens % sequences : tokens)) return TWA_ERR_INVALID_ARG;
  if (starts && twa_misaligned_to(starts, twa_itype_size(s_type))) return TWA_ERR_MISALIGNED;
  // blocks of a launch
  if (static_cast<long long>(sequences) * twa_ceil_div(channels, SCAN_CHANNELS) > 0x7FFFFFFFLL) return TWA_ERR_UNSUPPORTED;
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
  const bool packs = channels % 2 == 0 && scan_packs(x, ldx, size) && scan_packs(f, ldf, size) && scan_packs(h, ldh, size);
  const bool brief = tokens <= 2LL * SEG * sequences;
  if (dtype == TWA_BF16) scan_launch<bf16>(ctx, a, false, packs, brief);
  else scan_launch<float>(ctx, a, false, packs, brief);
  TWA_CUDA_OK(ctx, cudaGetLastError());
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
  const bool packs = channels % 2 == 0 && scan_packs(dh, lddh, size) && scan_packs(x, ldx, size) && scan_packs(f, ldf, size) &&
                     scan_packs(dx, lddx, size) && scan_packs(df, lddf, size);
  const bool brief = tokens <= 2LL * SEG * sequences;
  if (dtype == TWA_BF16) scan_launch<bf16>(ctx, a, true, packs, brief);
  else scan_launch<float>(ctx, a, true, packs, brief);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
