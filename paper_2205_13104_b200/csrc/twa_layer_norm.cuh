// Shared by the two directions of layer norm: arguments, the place of rows and columns, weights in shared memory.  sm_100a only.
#pragma once

#include "twa_ops.cuh"

namespace {

constexpr int LN_MAX_BLOCKS = 592;     // (a multiple of 8) blocks of the backward pass at most: rows of partial sums in the workspace
constexpr int LN_WARP_THREADS = 128;   // a warp or less per row: threads of a block at most
constexpr int LN_BLOCK_THREADS = 512;  // a block per row: at most
constexpr int LN_WIDE_THREADS = 1024, LN_WIDE_HELD = 16;
constexpr int LN_LOOP_THREADS = 512;   // rows wider than the registers of a block
constexpr int LN_LOOP_PARTS = 64;      // and the rows of partial sums for those

struct LnArgs {
  const void* x;
  const void* dy;      // backward
  void* y;             // forward: y; backward: dx
  const void* w;
  const void* b;
  float* mean;
  float* rstd;
  float* part;         // backward: [blocks][2][cols] partial sums of dw and db
  long long ldx, lddy, ldy, rows;
  int cols, w_dtype;
  int log_lanes;       // a warp per row or less: log2 of the threads of a row
  int log_classes;     // rows lie in 2^log_classes ways on 16-byte boundaries; a block takes rows of one
  float eps;
  unsigned long long wait_limit_ns;
  int* status;
};

// Sum over the threads of a row, PER <= 32.
template <int PER>
__device__ __forceinline__ float ln_sum_lanes(float v, int log_lanes) {
  if constexpr (PER != 0) {
    return twa_warp_sum(v);
  } else {
    for (int o = 0; o < log_lanes; ++o) v += __shfl_xor_sync(0xffffffffu, v, 1 << o);
    return v;
  }
}

// Sums of a (lanes 0 .. 15) and b (lanes 16 .. 31) over a warp: after the first step each half goes on with one of them.
__device__ __forceinline__ float ln_two_sums(float a, float b) {
  const bool upper = threadIdx.x & 16;
  float v = upper ? b : a;
  v += __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
  for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sums of v[0] and v[1] over the block of WARPS warps (0: as it was launched), one barrier.  What follows the barrier is the
// longest chain of a row: with the warps known it is two loads (gradient of 16384 x 2048 bfloat16: 39.4 us, with a loop and ten
// shuffles instead of five 48.3), for 32 warps a loop is better (2048 x 12000: 67.7 us, unrolled 76.2). `red` is used in turn by
// successive calls, two sets, so that a set is written again only after the next barrier.
template <int WARPS>
__device__ __forceinline__ void ln_block_sums(float (&v)[2], float (*red)[32][2], int& turn) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float mine = ln_two_sums(v[0], v[1]);
  float(*set)[2] = red[turn];
  turn ^= 1;
  if ((lane & 15) == 0) set[warp][lane >> 4] = mine;
  __syncthreads();
  v[0] = v[1] = 0.0f;
  if constexpr (WARPS != 0) {
#pragma unroll
    for (int w = 0; w < WARPS; w += 2) {
      const float4 q = *reinterpret_cast<const float4*>(set[w]);
      v[0] = v[0] + q.x + q.z;
      v[1] = v[1] + q.y + q.w;
    }
  } else {
    const int warps = blockDim.x >> 5;
    for (int w = 0; w < warps; ++w) {
      v[0] += set[w][0];
      v[1] += set[w][1];
    }
  }
}

// PER: threads of a row.  32: a warp; more: a block of so many; 0: a part of a warp, 2^log_lanes threads.  With PER known all
// of a thread's addresses are constants apart (16384 x 2048 bfloat16: 918 instructions a row against 570, 32 us against 26).
template <int PER>
constexpr int LN_THREADS = PER > 32 ? PER : LN_WARP_THREADS;      // of a block

// Which rows and columns a thread works on.  Rows: r = first + i * step, all with the same place on 16-byte boundaries.
// Columns: units of E elements counted from the 16-byte boundary at or below the row, unit k * per + t for k = 0, 1, ..;
// `skew` elements of the first unit lie before the row.
template <int E, int NV, int PER, bool FULL>
struct LnPlace {
  int lanes, t, group;        // PER == 0: threads of a row; this one's number; rows from the warp's first to this one's
  long long first, step;
  int skew, row_units, cols;
  __device__ __forceinline__ LnPlace(const LnArgs& a, int size) {
    const int classes = FULL ? 1 : 1 << a.log_classes, cls = FULL ? 0 : blockIdx.x & (classes - 1);
    const int block = FULL ? blockIdx.x : blockIdx.x >> a.log_classes, blocks = FULL ? gridDim.x : gridDim.x >> a.log_classes;
    long long q;
    if (PER <= 32) {
      const int lane = threadIdx.x & 31, log_lanes = PER ? 5 : a.log_lanes, groups = 32 >> log_lanes, warps = LN_WARP_THREADS / 32;
      lanes = 1 << log_lanes;
      t = lane & (lanes - 1);
      group = lane >> log_lanes;
      q = (static_cast<long long>(block) * warps + (threadIdx.x >> 5)) * groups;
      step = static_cast<long long>(blocks) * warps * groups * classes;
    } else {
      lanes = PER;
      t = threadIdx.x;
      group = 0;
      q = block;
      step = static_cast<long long>(blocks) * classes;
    }
    first = q * classes + cls;
    group *= classes;
    cols = a.cols;
    skew = FULL || E == 1 ? 0 : static_cast<int>(((reinterpret_cast<uintptr_t>(a.x) + cls * a.ldx * size) & 15) / size);
    row_units = (skew + cols + E - 1) / E;
  }
  // units of the vectors in shared memory: all that the threads can have
  __device__ __forceinline__ int units() const { return (PER ? PER : lanes) * NV; }
  __device__ __forceinline__ int unit(int k) const { return k * (PER ? PER : lanes) + t; }
  __device__ __forceinline__ bool in(int k) const { return FULL || unit(k) < row_units; }
  __device__ __forceinline__ int column(int k, int e) const { return unit(k) * E + e - skew; }
  __device__ __forceinline__ bool valid(int k, int e) const {
    return FULL || (E == 1 ? in(k) : column(k, e) >= 0 && column(k, e) < cols);
  }
  // every element of the unit in the row
  __device__ __forceinline__ bool whole(int k) const {
    return FULL || (E == 1 ? in(k) : unit(k) * E >= skew && (unit(k) + 1) * E <= skew + cols);
  }
  // The unit of the row that begins at `row`.  Of a unit that the row has in part, elements outside are what is beside the row in
  // memory (`inner`: there are rows before and after it, E - 1 elements apart at least, see ln_classes), or 0.
  template <typename T>
  __device__ __forceinline__ void load(twa_pack<T, E>& p, const T* row, int k, bool inner) const {
    if (E == 1 || inner || whole(k)) {
      p.load(row - skew + unit(k) * E);
    } else {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = valid(k, e) ? twa_to_float(row[column(k, e)]) : 0.0f;
      p.from(v);
    }
  }
  // 0 for what is not of the row
  __device__ __forceinline__ void keep_valid(int k, float* v) const {
    if constexpr (!FULL) {
      if (whole(k)) return;
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = valid(k, e) ? v[e] : 0.0f;
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, int k, const float* v) const {
    if (whole(k)) {
      twa_pack<T, E>::store(row - skew + unit(k) * E, v);
    } else if constexpr (E > 1) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (valid(k, e)) row[column(k, e)] = twa_from_float<T>(v[e]);
    }
  }
};

extern __shared__ __align__(16) float ln_planes[];
// A vector of float32 per column in shared memory, by units of E elements; E == 8: in two planes of half a unit each so that
// 16-byte accesses of neighbouring threads do not collide.
template <int E>
struct LnPlane {
  static constexpr int HALF = E == 8 ? 4 : E;
  int from, units;             // its place in ln_planes
  __device__ __forceinline__ int at(int unit, int e) const { return from + (e / HALF * units + unit) * HALF + e % HALF; }
  __device__ __forceinline__ void load(int unit, float* v) const {
#pragma unroll
    for (int e = 0; e < E; e += HALF) {
      if constexpr (HALF == 4) {
        const float4 q = *reinterpret_cast<const float4*>(&ln_planes[at(unit, e)]);
        v[e] = q.x; v[e + 1] = q.y; v[e + 2] = q.z; v[e + 3] = q.w;
      } else {
        v[e] = ln_planes[at(unit, e)];
      }
    }
  }
  __device__ __forceinline__ void store(int unit, const float* v) const {
#pragma unroll
    for (int e = 0; e < E; e += HALF) {
      if constexpr (HALF == 4) *reinterpret_cast<float4*>(&ln_planes[at(unit, e)]) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
      else ln_planes[at(unit, e)] = v[e];
    }
  }
};
// Fills it from a vector of any type and alignment whose element 0 is `skew` elements into the first unit, or with `missing`;
// LN_STAGE loads of a thread are under way at once.
constexpr int LN_STAGE = 16;
template <int E>
__device__ __forceinline__ void ln_stage(const LnPlane<E>& to, const void* from, int dtype, int skew, int cols, float missing) {
  const int n = to.units * E;
  for (int c0 = threadIdx.x; c0 < n; c0 += LN_STAGE * blockDim.x) {
    float v[LN_STAGE];
#pragma unroll
    for (int i = 0; i < LN_STAGE; ++i) {
      const int c = c0 + i * blockDim.x - skew;
      v[i] = from && c >= 0 && c < cols ? twa_load_any(from, dtype, c) : missing;
    }
#pragma unroll
    for (int i = 0; i < LN_STAGE; ++i) {
      const int c = c0 + i * blockDim.x;
      if (c < n) ln_planes[to.at(c / E, c % E)] = v[i];
    }
  }
}

// The NV * E elements of a thread as pairs.
template <int E, int NV>
struct LnPairs {
  static constexpr int N = E * NV, P = (N + 1) / 2;
  static __device__ __forceinline__ twa_f2 get(const float* v, int i) { return twa_pair(v[2 * i], 2 * i + 1 < N ? v[2 * i + 1] : 0.0f); }
  static __device__ __forceinline__ void put(float* v, int i, twa_f2 p) {
    float lo, hi;
    twa_unpair(p, lo, hi);
    v[2 * i] = lo;
    if (2 * i + 1 < N) v[2 * i + 1] = hi;
  }
};

typedef void (*LnKernel)(LnArgs);
struct LnPlan {
  LnKernel kernel;                 // null: the rows do not fit a block
  int threads, blocks, log_lanes;  // threads of a block, blocks, log2 of the threads of a row where those are in one warp
  int log_classes;
  size_t smem;
};

// Ways in which the rows of all matrices lie on 16-byte boundaries, if they do alike; else 0, and the rows are read element by
// element.  So are rows that begin less than a unit of 16 bytes apart but for one element: a row's first and last unit reach up to
// that far beside it, which then is more than a neighbouring row (3 x 2 bfloat16: row 1's unit is 8 of the matrix's 6 elements).
int ln_classes(const void* p, long long ld, const void* q, long long ldq, const void* s, long long lds, long long rows, int cols,
               size_t size) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p) & 15;
  const long long d = (ld * static_cast<long long>(size)) & 15;
  if ((reinterpret_cast<uintptr_t>(q) & 15) != a || (reinterpret_cast<uintptr_t>(s) & 15) != a) return 0;
  const long long unit = 16 / static_cast<long long>(size);
  if (rows > 1 && (ld < unit - 1 || ldq < unit - 1 || lds < unit - 1)) return 0;
  if (rows > 1 && (((ldq * static_cast<long long>(size)) & 15) != d || ((lds * static_cast<long long>(size)) & 15) != d)) return 0;
  if (a == 0 && (d == 0 || rows <= 1) && cols * size % 16 == 0) return 1;
  return static_cast<int>(16 / size);
}

int ln_check(const twa_ctx* ctx, twa_dtype dt, twa_dtype wt, int64_t rows, int cols) {
  if (!ctx || !twa_dtype_ok(dt) || !twa_dtype_ok(wt) || rows < 0 || cols < 1) return TWA_ERR_INVALID_ARG;
  if (rows > (1LL << 40) || cols > TWA_LAYER_NORM_MAX_COLS) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

// ---- plans.  The directions (LnForward, LnBackward) differ in
//   HELD<E, PER>    elements that a thread holds of a row at most
//   MAX_BLOCKS      blocks at most
//   kernel<..>()    the kernel of NV units a thread; full: the row is exactly the units of its threads
//   ring_bytes()    shared memory of the rows under way
//   wide<..>()      the plan of rows on 16-byte boundaries that are too wide for those kernels, where there is one

// The kernel that holds at least nv units a thread, and how many that is.
template <typename Dir, typename T, int E, int PER>
LnKernel ln_pick(int* nv, int units, bool aligned) {
  const int wanted = *nv;
  constexpr int held = Dir::template HELD<E, PER>;
#define LN_TRY(n, if_more)                                                              \
  if constexpr (E * n <= held && (PER <= 32 || 2 * E * n >= held) && (if_more)) {       \
    if (wanted <= n) {                                                                  \
      *nv = n;                                                                          \
      return Dir::template kernel<T, E, n, PER>(aligned, units == PER * n);             \
    }                                                                                   \
  }
  LN_TRY(1, true)
  LN_TRY(2, true)
  LN_TRY(3, E > 1 && PER > 0)
  LN_TRY(4, true)
  LN_TRY(6, E > 1 && PER > 0)
  LN_TRY(8, true)
  LN_TRY(16, true)
  LN_TRY(32, true)
#undef LN_TRY
  return nullptr;
}

template <typename Dir, typename T, int E>
int ln_plan_units(twa_ctx* ctx, int classes, long long rows, int cols, LnPlan* plan) {
  // with several classes a row can begin anywhere in its first unit
  const int units = (cols + E - 1) / E + (classes > 1 ? 1 : 0);
  constexpr int warp_held = Dir::template HELD<E, 32> / E, held = Dir::template HELD<E, 64> / E;
  const bool aligned = classes == 1;
  LnPlan p = {nullptr, 0, 0, 5, 0, 0};
  while (1 << p.log_classes < classes) ++p.log_classes;
  int nv = 0, per = 32;
  long long blocks = rows;
  p.threads = LN_WARP_THREADS;
  if (units <= 32 * warp_held) {
    // as few threads a row as hold it, while there are rows enough to keep the SMs busy
    while (p.log_lanes > 0 && units <= held << (p.log_lanes - 1) && (rows << (p.log_lanes - 1)) >= 32LL * 16 * ctx->sm_count) --p.log_lanes;
    while (p.log_lanes > 0 && units <= 1 << (p.log_lanes - 1)) --p.log_lanes;
    per = 1 << p.log_lanes;
    nv = (units + per - 1) / per;
    p.kernel = per == 32 ? ln_pick<Dir, T, E, 32>(&nv, units, aligned) : ln_pick<Dir, T, E, 0>(&nv, units, aligned);
    blocks = twa_ceil_div(rows, p.threads / per);
  } else if (units <= LN_BLOCK_THREADS * held) {
    for (per = 64; units > per * held;) per *= 2;
    nv = (units + per - 1) / per;
    p.threads = per;
    p.kernel = per == 64 ? ln_pick<Dir, T, E, 64>(&nv, units, aligned)
               : per == 128 ? ln_pick<Dir, T, E, 128>(&nv, units, aligned)
               : per == 256 ? ln_pick<Dir, T, E, 256>(&nv, units, aligned) : ln_pick<Dir, T, E, 512>(&nv, units, aligned);
  }
  p.smem = sizeof(float) * 2 * per * nv * E + (E > 1 ? Dir::ring_bytes(per, nv, aligned) : 0);
  if (!p.kernel && aligned) Dir::template wide<T, E>(units, &p);
  if (p.kernel && p.smem > 44 * 1024) {      // 48 KB with what the kernel declares
    // which of the kernels that can need as much: by threads of a row (0: the one of rows too wide for the others) and units of a thread
    static int smem_set[6][40][3][64] = {};
    int log = nv ? 1 : 0;
    while (nv && 16 << log < per) ++log;
    int rc = twa_ensure_smem(ctx, reinterpret_cast<const void*>(p.kernel),
                             &smem_set[log][nv][aligned ? (units == per * nv ? 2 : 1) : 0][ctx->device & 63], static_cast<int>(p.smem));
    if (rc) return rc;
  }
  const long long per_sm = p.threads < 512 ? 512 / p.threads : 1;
  long long most = ctx->sm_count * per_sm;
  if (most > Dir::MAX_BLOCKS) most = Dir::MAX_BLOCKS;
  if (blocks > most) blocks = most;
  if (classes > 1) blocks = twa_ceil_div(blocks, classes) * classes;
  p.blocks = static_cast<int>(blocks);
  *plan = p;
  return TWA_OK;
}

// classes: ways in which the rows lie on 16-byte boundaries (1: all begin on one), 0: they are read element by element.
template <typename Dir, typename T>
int ln_plan(twa_ctx* ctx, int classes, long long rows, int cols, LnPlan* plan) {
  if (classes) {
    int rc = ln_plan_units<Dir, T, twa_vec<T>>(ctx, classes, rows, cols, plan);
    if (rc || plan->kernel) return rc;
  }
  return ln_plan_units<Dir, T, 1>(ctx, 1, rows, cols, plan);
}

}  // namespace
