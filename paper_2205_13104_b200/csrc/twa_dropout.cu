// Dropout whose mask is never stored, and its gradient.
//
//   y = residual + [u >= t] x 65536 / (65536 - t),   t = round(65536 p)
//
// u are 16 bits of a counter-based generator, Philox4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011): a round multiplies two words of the counter by constants and adds the key's halves, which
// go up by constants from round to round.  The counter is (column / 8, row, site, step), the key the seed: a call's 128 bits
// are the numbers of 8 neighbouring columns, and the backward pass draws them again from the same place.
//
// Bound by memory with a residual: 32768 x 2048 bfloat16 59 us in a row of calls (403 MB, 6.9 TB/s: two thirds are loads, which are
// faster than the halves of a copy; a single call leaves some 50 MB of its stores in L2 and moves 351 MB at 6.4 TB/s, 80 % of DRAM's
// peak); without one 43 us (268 MB, 6.3 TB/s), where the generator's products count: some 60 instructions a call of it, the key's
// additions shared by a thread's two calls (47 us for a single call, 53 when they are apart).
// 16 bits an element halve it against 32; a probability is then a multiple of 2^-16, and the scale is that of the multiple.
// Rows between 16-byte boundaries go by the element and find their bit in another lane: 32768 x 2047 bfloat16 84 us with a residual,
// 67 without (a single call 93 and 73), bound by instructions (two elements an access, where rows lie alike between words: 88 and 88).
#include "twa_ops.cuh"

namespace {

constexpr int DROP_THREADS = 256;

// n / d for n < 2^31: (n m) >> shift with m = ceil(2^shift / d), shift = 31 + ceil(log2 d).  m exceeds 2^shift / d by less than
// one, the product by less than n / 2^31 2^-ceil(log2 d) <= 1 / d of the result, which does not reach the next integer.
struct Divisor {
  uint32_t d, m;
  int shift;
  explicit Divisor(uint32_t by) : d(by) {
    int log = 0;
    while ((1ULL << log) < d) ++log;
    shift = 31 + log;
    m = static_cast<uint32_t>(((1ULL << shift) + d - 1) / d);
  }
  __device__ __forceinline__ uint32_t divide(uint32_t n) const {
    return static_cast<uint32_t>((static_cast<unsigned long long>(n) * m) >> shift);
  }
};

struct DropArgs {
  const void* x;
  const void* residual;
  void* y;
  const unsigned long long* rng;     // seed, step
  long long ldx, ldr, ldy;
  unsigned rows, row0;               // of this launch, and the first one's number
  int cols;
  uint32_t site, threshold;          // threshold: t << 16
  float scale;
  Divisor parts;                     // of a row
};

struct Words {
  uint32_t w[4];
};
// For N counters at once: the key's halves are the same for all.
template <int N>
__device__ __forceinline__ void philox(Words (&u)[N], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t* c = u[i].w;
      const unsigned long long p0 = static_cast<unsigned long long>(c[0]) * 0xD2511F53u, p1 = static_cast<unsigned long long>(c[2]) * 0xCD9E8D57u;
      c[0] = static_cast<uint32_t>(p1 >> 32) ^ c[1] ^ k0;
      c[2] = static_cast<uint32_t>(p0 >> 32) ^ c[3] ^ k1;
      c[1] = static_cast<uint32_t>(p1);
      c[3] = static_cast<uint32_t>(p0);
    }
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}
// Whether element e of the eight is kept.
__device__ __forceinline__ bool drop_keeps(const Words& u, int e, uint32_t threshold) {
  return (e & 1 ? u.w[e >> 1] : u.w[e >> 1] << 16) >= threshold;
}

// Eight columns a unit, on 16-byte boundaries; DROP_UNITS units a thread.  The generator needs nothing from memory but the
// seed, so it runs while the loads are under way.
constexpr int DROP_UNITS = 2;
template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(DROP_THREADS) dropout_kernel(DropArgs a) {
  twa_begin(a.x, a.residual, a.rng);
  constexpr int V = twa_vec<T>, N = 8 / V;
  const T* x = static_cast<const T*>(a.x);
  const T* res = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  const unsigned long long seed = __ldg(a.rng), step = __ldg(a.rng + 1);
  const unsigned total = a.rows * a.parts.d;
  const unsigned first = blockIdx.x * (DROP_THREADS * DROP_UNITS) + threadIdx.x;
  twa_pack<T, V> raw[DROP_UNITS][N], add[DROP_UNITS][N];
  unsigned row[DROP_UNITS], unit[DROP_UNITS];
#pragma unroll
  for (int k = 0; k < DROP_UNITS; ++k) {
    const unsigned n = first + k * DROP_THREADS;
    row[k] = a.parts.divide(n);
    unit[k] = n - row[k] * a.parts.d;
    if (n >= total) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      raw[k][i].load(x + row[k] * a.ldx + unit[k] * 8 + i * V);
      if (RESIDUAL) add[k][i].load(res + row[k] * a.ldr + unit[k] * 8 + i * V);
    }
  }
  Words u[DROP_UNITS];
#pragma unroll
  for (int k = 0; k < DROP_UNITS; ++k) u[k] = {{unit[k], a.row0 + row[k], a.site, static_cast<uint32_t>(step)}};
  philox(u, static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
#pragma unroll
  for (int k = 0; k < DROP_UNITS; ++k) {
    if (first + k * DROP_THREADS >= total) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float v[V], r[V];
      raw[k][i].widen(v);
      if (RESIDUAL) add[k][i].widen(r);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float kept = RESIDUAL ? fmaf(v[e], a.scale, r[e]) : v[e] * a.scale;
        v[e] = drop_keeps(u[k], i * V + e, a.threshold) ? kept : (RESIDUAL ? r[e] : 0.0f);
      }
      twa_pack<T, V>::store(y + row[k] * a.ldy + unit[k] * 8 + i * V, v);
    }
  }
}

// Rows on any boundary: a warp takes DROP_UNITS x 256 columns.  Each lane draws the numbers of eight neighbouring columns and keeps one
// bit of each; elements go by lane, so that accesses are contiguous, and find their bit in another lane.
constexpr int DROP_PART = DROP_UNITS * 256;
template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(DROP_THREADS) dropout_any_kernel(DropArgs a) {
  twa_begin(a.x, a.residual, a.rng);
  const unsigned task = blockIdx.x * (DROP_THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (task >= a.rows * a.parts.d) return;
  const unsigned row = a.parts.divide(task), part = task - row * a.parts.d;
  const int left = a.cols - static_cast<int>(part) * DROP_PART - static_cast<int>(lane);
  const T* x = static_cast<const T*>(a.x) + row * a.ldx + part * DROP_PART + lane;
  const T* res = static_cast<const T*>(a.residual) + (RESIDUAL ? row * a.ldr + part * DROP_PART + lane : 0);
  T* y = static_cast<T*>(a.y) + row * a.ldy + part * DROP_PART + lane;
  twa_pack<T, 1> raw[DROP_UNITS * 8], add[DROP_UNITS * 8];
#pragma unroll
  for (int k = 0; k < DROP_UNITS * 8; ++k)
    if (k * 32 < left) {
      raw[k].load(x + k * 32);
      if (RESIDUAL) add[k].load(res + k * 32);
    }
  const unsigned long long seed = __ldg(a.rng), step = __ldg(a.rng + 1);
  Words u[DROP_UNITS];
#pragma unroll
  for (int i = 0; i < DROP_UNITS; ++i) u[i] = {{(part * DROP_UNITS + i) * 32 + lane, a.row0 + row, a.site, static_cast<uint32_t>(step)}};
  philox(u, static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
#pragma unroll
  for (int i = 0; i < DROP_UNITS; ++i) {
    unsigned bits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (drop_keeps(u[i], e, a.threshold)) bits |= 1u << e;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool keep = __shfl_sync(0xffffffffu, bits, 4 * k + (lane >> 3)) >> (lane & 7) & 1;
      const int n = i * 8 + k;
      if (n * 32 >= left) continue;
      float v, r = 0.0f;
      raw[n].widen(&v);
      if (RESIDUAL) add[n].widen(&r);
      y[n * 32] = twa_from_float<T>(keep ? fmaf(v, a.scale, r) : r);
    }
  }
}

bool drop_packs(const void* p, long long ld, size_t size) { return !twa_misaligned_to(p, 16) && ld * size % 16 == 0; }

template <typename T>
void drop_launch(twa_ctx* ctx, DropArgs a, int64_t rows) {
  const size_t size = sizeof(T);
  const bool packs = a.cols % 8 == 0 && drop_packs(a.x, a.ldx, size) && drop_packs(a.y, a.ldy, size) &&
                     (!a.residual || drop_packs(a.residual, a.ldr, size));
  a.parts = Divisor(static_cast<uint32_t>(packs ? a.cols / 8 : twa_ceil_div(a.cols, DROP_PART)));
  // tasks of a launch are counted in 31 bits
  const long long most = ((1LL << 31) - DROP_THREADS * DROP_UNITS) / a.parts.d;
  for (long long r = 0; r < rows; r += most) {
    a.row0 = static_cast<unsigned>(r);
    a.rows = static_cast<unsigned>(rows - r < most ? rows - r : most);
    const long long tasks = static_cast<long long>(a.rows) * a.parts.d;
    auto launch = [&](auto kernel, int tasks_a_block) {
      twa_launch(ctx->stream, kernel, static_cast<unsigned>(twa_ceil_div(tasks, tasks_a_block)), DROP_THREADS, 0, a);
    };
    constexpr int WARPS = DROP_THREADS / 32;
    if (packs) a.residual ? launch(dropout_kernel<T, true>, DROP_THREADS * DROP_UNITS) : launch(dropout_kernel<T, false>, DROP_THREADS * DROP_UNITS);
    else a.residual ? launch(dropout_any_kernel<T, true>, WARPS) : launch(dropout_any_kernel<T, false>, WARPS);
    a.x = static_cast<const T*>(a.x) + most * a.ldx;
    a.y = static_cast<T*>(a.y) + most * a.ldy;
    if (a.residual) a.residual = static_cast<const T*>(a.residual) + most * a.ldr;
  }
}

}  // namespace

extern "C" {

int twa_dropout(twa_ctx* ctx, const void* x, int64_t ldx, twa_dtype dtype, int64_t rows, int cols, float p, const int64_t* rng,
                int64_t site, const void* residual, int64_t ldr, void* y, int64_t ldy) {
  if (!ctx || !twa_dtype_ok(dtype) || rows < 0 || cols < 1 || !(p >= 0.0f && p < 1.0f)) return TWA_ERR_INVALID_ARG;
  if (site < 0 || site > 0xFFFFFFFFLL) return TWA_ERR_INVALID_ARG;
  if (rows > TWA_DROPOUT_MAX_ROWS || cols > TWA_DROPOUT_MAX_COLS) return TWA_ERR_UNSUPPORTED;
  if (rows == 0) return TWA_OK;
  if (!x || !y || !rng || ldx < cols || ldy < cols || (residual && ldr < cols)) return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(x, size) || twa_misaligned_to(y, size) || twa_misaligned_to(residual, size) || twa_misaligned_to(rng, 8))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  int t = static_cast<int>(rint(static_cast<double>(p) * 65536.0));
  if (t > 65535) t = 65535;
  DropArgs a = {x, residual, y, reinterpret_cast<const unsigned long long*>(rng), ldx, ldr, ldy, 0, 0, cols, static_cast<uint32_t>(site),
                static_cast<uint32_t>(t) << 16, static_cast<float>(65536.0 / (65536 - t)), Divisor(1)};
  if (dtype == TWA_BF16) drop_launch<bf16>(ctx, a, rows);
  else drop_launch<float>(ctx, a, rows);
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

int twa_dropout_backward(twa_ctx* ctx, const void* dy, int64_t lddy, twa_dtype dtype, int64_t rows, int cols, float p, const int64_t* rng,
                         int64_t site, void* dx, int64_t lddx) {
  return twa_dropout(ctx, dy, lddy, dtype, rows, cols, p, rng, site, nullptr, 0, dx, lddx);
}

}  // extern "C"
