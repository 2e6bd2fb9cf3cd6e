// Log probabilities of given tokens with the entropy of their distribution and its most likely tokens, and the
// gradient of both.  For a row z of logits, p = softmax(z):
//
//   forward    lse = log sum exp z,  logp = z[target] - lse,  H = lse - sum p z = log S - A / S
//              with m = max z, S = sum exp(z - m), A = sum exp(z - m) (z - m)
//   backward   dz[j] = d_logp ([j == target] - p[j]) - d_H p[j] (log p[j] + H)
//
// Both are bound by memory: forward reads the logits once, backward reads and writes them once.
//
// Forward: a block streams its rows through a ring of bulk copies.  One warp issues the copies, eight add up, and two
// finish, even and odd rows in turn: they take the eight warps' results of a row while those are at the next ones, so
// that neither memory nor the sums wait for the merges, the search and the stores at the end of a row.  Every summing thread keeps the running m, S and A of the elements it meets (S and A are
// rescaled when m grows); the threads' triples are merged at the end of the row.  The arithmetic has to stay below five
// instructions an element to keep up with memory in bfloat16: exponents are one packed multiply-add,
// d = z log2 e - c with c = m log2 e as rounded (the rounding error is known and taken out of S and A at the end), one
// ex2 each, and packed sums.  -inf would make p d = 0 * -inf: values are raised to -2^126 first (p is 0 there either way).
// c loses its digits when m is far from zero, so it is held within +-8192 log2 e; a row (or a block's part of one) whose
// maximum lies beyond is summed once more with differences to that maximum taken first.
//
// The most likely tokens cost no second pass.  With T the k-th largest of the maxima of 32 groups of threads, k elements
// are T or more, so each of the k best elements is, and lies with a thread whose maximum is.  Each thread also leaves the
// maxima of its parts of the row (SLOTS of them): only the parts of those threads that reach T (some 1.5 k) are
// looked at again, in L2, and the few elements of T or more are sorted by (value, smaller index first).
//
// 8192 x 50272 bfloat16 with entropy and 5 tokens: 162 to 178 us (by the SM clock), 4.6 to 5.1 TB/s, bound by the sums' chains (issue
// slots 63 % in use, the unit for exponentials 56 %, with 19 warps an SM); 333 x 32003 float32 with 20 tokens 19 us (43 MB): a
// little more than a row a block, whose end nothing hides.  Where fewer groups than `top` have a token above -inf every
// thread's parts are candidates, and a warp looks at the whole row again: 8192 rows with 20 tokens 174 us with 300 of 50272 tokens
// allowed, 2980 us with 30.  Backward 8192 x 50272: 264 to 278 us, 5.9 to 6.2 TB/s.
#include "twa_ops.cuh"

namespace {

constexpr int LP_WARPS = 8, LP_THREADS = LP_WARPS * 32;     // threads that add up
constexpr int LP_COPY = LP_WARPS, LP_FINISH = LP_WARPS + 1; // the warp that issues copies, the first that finishes rows
constexpr int LP_FINISHERS = 2;
constexpr int LP_BLOCK = LP_THREADS + 32 * (1 + LP_FINISHERS);
constexpr int LP_PER_THREAD = 4;                            // 16-byte units of a thread in a chunk
constexpr int LP_CHUNK = LP_THREADS * LP_PER_THREAD;        // units
// Without the search three blocks fit an SM's registers, with it two (8192 x 50272 bfloat16 with entropy: without tokens 140 us
// and 148 with two; with 5 tokens 162 us, with three 165 to 199).
template <bool TOP>
constexpr int LP_BLOCKS_PER_SM = TOP ? 2 : 3;
template <bool TOP>
constexpr int LP_STAGES = TOP ? 4 : 3;
constexpr int LP_SLOTS = 16;                                // parts of a row whose maxima a thread leaves
constexpr int LP_BUFFER = 128;                              // candidates that are sorted without a further look
constexpr int LP_MAX_CLUSTER = 8;
// Blocks an SM up to which rows are split over clusters (148 rows of 50272 split in two 16 us; beyond it, with four blocks an SM,
// 30 us).
constexpr long long LP_SPLIT_ROWS = 2;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LP_FAR = 8192.0f;                           // bound of what exponents are taken against
typedef unsigned long long u64;

__device__ __forceinline__ float lp_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The four words of a 16-byte unit: the maximum of the elements of two words, elements raised to -2^126 (NaN stays), a
// word's elements widened to pairs of floats.
template <typename T>
struct LpWord;
template <>
struct LpWord<bf16> {
  static constexpr uint32_t NONE = 0xff80ff80u;              // -inf twice
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float max1(uint32_t a) { return fmaxf(twa_bf16_lo(a), twa_bf16_hi(a)); }
  static __device__ __forceinline__ uint32_t raise(uint32_t a) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0xfe80fe80u));
    return r;
  }
  static constexpr int PAIRS = 4;                            // of a unit
  static __device__ __forceinline__ u64 pair(const uint32_t* w, int i) { return twa_pair(twa_bf16_lo(w[i]), twa_bf16_hi(w[i])); }
};
template <>
struct LpWord<float> {
  static constexpr uint32_t NONE = 0xff800000u;
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
  static __device__ __forceinline__ float max1(uint32_t a) { return __uint_as_float(a); }
  static __device__ __forceinline__ uint32_t raise(uint32_t a) {
    uint32_t r;
    asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0xfe800000u));
    return r;
  }
  static constexpr int PAIRS = 2;
  static __device__ __forceinline__ u64 pair(const uint32_t* w, int i) {
    return twa_pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  }
};

// Order-preserving bits of a value; zeros of both signs are equal.  0 is below every value, -inf included.
__device__ __forceinline__ uint32_t lp_rank(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float lp_unrank(uint32_t r) {
  return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r);
}
__device__ __forceinline__ u64 lp_key(float v, uint32_t place) { return static_cast<u64>(lp_rank(v)) << 32 | (0xffffffffu - place); }

// A row as 16-byte units counted from the aligned address at or below its first element.  The units that lie wholly in
// it are first .. first + whole - 1; the elements before and after them (at most E - 1 each) are read one by one.
template <typename T>
struct LpRow {
  static constexpr int E = twa_vec<T>;
  const T* base;       // unit 0, element 0 (may lie before the row)
  int skew, cols;      // the row's element j is base[skew + j]
  int first, whole;
  __device__ __forceinline__ LpRow(const T* row, int n) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row);
    skew = static_cast<int>((a & 15) / sizeof(T));
    base = reinterpret_cast<const T*>(a & ~static_cast<uintptr_t>(15));
    cols = n;
    first = skew ? 1 : 0;
    whole = max(0, (skew + cols) / E - first);
  }
  // first of the whole units of part p of 2^log_parts
  __device__ __forceinline__ int part_from(int p, int log_parts) const {
    return static_cast<int>(static_cast<unsigned long long>(whole) * p >> log_parts);
  }
  // elements before the whole units, and after them
  __device__ __forceinline__ int head() const { return min(cols, first * E - skew); }
  __device__ __forceinline__ int tail_from() const { return min(cols, (first + whole) * E - skew); }
};

// Sums of some elements of a row: m = their maximum (-inf: none above -inf), with d = (z - m) log2 e
// s = sum 2^d, a = sum 2^d d.
struct LpStat {
  float m, s, a;
};
// The base of a thread's sums.
__device__ __forceinline__ float lp_base(float m) { return fminf(fmaxf(m, -LP_FAR), LP_FAR); }
// Sums relative to lp_base(m) of groups of LANES neighbouring lanes, of the maximum of all 32 in every lane.
template <bool ENT, int LANES>
__device__ __forceinline__ LpStat lp_merge_near(const LpStat& x) {
  LpStat r;
  r.m = lp_unrank(__reduce_max_sync(0xffffffffu, lp_rank(x.m)));
  const float d = fmaxf((lp_base(x.m) - lp_base(r.m)) * LOG2E, -150.0f), f = lp_exp2(d);
  r.s = x.s * f;
  r.a = ENT ? f * (x.a + d * x.s) : 0.0f;
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
    if (ENT) r.a += __shfl_xor_sync(0xffffffffu, r.a, o);
  }
  return r;
}
// Sums relative to m (0 or NaN where m is -inf) of all lanes.
template <bool ENT>
__device__ __forceinline__ LpStat lp_merge(const LpStat& x) {
  LpStat r;
  r.m = lp_unrank(__reduce_max_sync(0xffffffffu, lp_rank(x.m)));
  const float base = r.m == -INFINITY ? 0.0f : r.m, d = fmaxf((x.m - base) * LOG2E, -150.0f), f = lp_exp2(d);
  r.s = twa_warp_sum(x.s * f);
  r.a = ENT ? twa_warp_sum(f * (x.a + d * x.s)) : 0.0f;
  return r;
}

// ---- sorting keys ------------------------------------------------------------------------------------
__device__ __forceinline__ u64 lp_shfl_xor(u64 v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }

// Sorts 32 keys of a warp, largest in lane 0 (bitonic network).
__device__ __forceinline__ u64 lp_sort32(u64 v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j; j >>= 1) {
      const u64 o = lp_shfl_xor(v, j);
      const bool keep_max = ((lane & j) == 0) == ((lane & k) == 0 || k == 32);
      v = keep_max ? (v > o ? v : o) : (v < o ? v : o);
    }
  return v;
}
// The 32 best of two sorted lists, sorted: `other` is lane's entry of the second list reversed.
__device__ __forceinline__ u64 lp_merge32(u64 v, u64 other_reversed) {
  const int lane = threadIdx.x & 31;
  v = v > other_reversed ? v : other_reversed;
#pragma unroll
  for (int j = 16; j; j >>= 1) {
    const u64 o = lp_shfl_xor(v, j);
    v = (lane & j) == 0 ? (v > o ? v : o) : (v < o ? v : o);
  }
  return v;
}
// The number of the warp's keys above `v`: its place in descending order, where keys differ.  32 independent comparisons
// against keys read from shared memory (`row`, the warp's own) take a third of the time of the network's 15 dependent steps.
template <typename K>
__device__ __forceinline__ int lp_place32(K v, K* row) {
  row[threadIdx.x & 31] = v;
  __syncwarp();
  int above = 0;
  if constexpr (sizeof(K) == 8) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(row + i);
      above += (o.x > v) + (o.y > v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(row + i);
      above += (o.x > v) + (o.y > v) + (o.z > v) + (o.w > v);
    }
  }
  __syncwarp();
  return above;
}
// Adds one key per lane to a sorted list of the 32 best.
__device__ __forceinline__ u64 lp_take32(u64 list, u64 key) {
  if (!__any_sync(0xffffffffu, key > __shfl_sync(0xffffffffu, list, 31))) return list;
  return lp_merge32(list, __shfl_xor_sync(0xffffffffu, lp_sort32(key), 31));
}

// The best 32 of the first `count` keys of a buffer of at least 32, sorted; the buffer is used up.
__device__ __forceinline__ u64 lp_sort_buffer(u64* buffer, int count) {
  const int lane = threadIdx.x & 31;
  u64 list = lane < count ? buffer[lane] : 0;
  if (count <= 32) {
    __syncwarp();
    const int place = lp_place32(list, buffer);
    buffer[lane] = 0;
    __syncwarp();
    if (list) buffer[place] = list;
    __syncwarp();
    return buffer[lane];
  }
  list = lp_sort32(list);
  for (int i = 32; i < count; i += 32) list = lp_take32(list, i + lane < count ? buffer[i + lane] : 0);
  return list;
}

struct LpArgs {
  const void* logits;
  const void* targets;
  float *logp, *lse, *entropy;
  int* top_ids;
  float* top_logp;
  const float *d_logp, *d_entropy;
  void* dlogits;
  long long ld, ldd, rows, ignore_id;
  int vocab, itype, top;
  unsigned long long wait_limit_ns;
  int* status;
};

template <bool TOP>
struct LpShared {
  uint4 ring[LP_STAGES<TOP>][LP_CHUNK];
  u64 full[LP_STAGES<TOP>], empty[LP_STAGES<TOP>];        // the ring's stages
  u64 row_full[LP_FINISHERS], row_empty[LP_FINISHERS];    // a row's results, by the warp that finishes it
  LpStat stat[LP_FINISHERS][LP_WARPS];
  uint32_t key[LP_FINISHERS][TOP ? LP_THREADS : 1];           // ranks of the threads' maxima, 0: no element
  float slot[LP_FINISHERS][TOP ? LP_SLOTS : 1][LP_THREADS];
  uint4 hit[LP_FINISHERS][TOP ? LP_BUFFER : 1]; // units with candidates, candidates
  alignas(16) u64 buffer[LP_FINISHERS][TOP ? LP_BUFFER : 2];
  alignas(16) uint32_t group[LP_FINISHERS][32];
  int hit_unit[LP_FINISHERS][TOP ? LP_BUFFER : 1];
  int pair[LP_FINISHERS][TOP ? LP_BUFFER : 1];  // slot and thread
  int chosen[LP_FINISHERS][TOP ? LP_THREADS : 1];
  u64 best[32];                                 // this block's best, read by the first block of the cluster
  LpStat mine;                                  // this block's sums, likewise
  int gave_up;
};

// By one warp, for rows that are out of the ordinary.  Sums over row[from .. to - 1] with differences to m taken first;
template <typename T, bool ENT>
__device__ __noinline__ LpStat lp_sum_far(const T* row, int from, int to, float m) {
  float s = 0.0f, w = 0.0f;
  for (int j = from + static_cast<int>(threadIdx.x & 31); j < to; j += 32) {
    const float d = (twa_to_float(row[j]) - m) * LOG2E, p = lp_exp2(d);
    s += p;
    if (ENT) w = fmaf(p, fmaxf(d, -150.0f), w);
  }
  return {m, twa_warp_sum(s), ENT ? twa_warp_sum(w) : 0.0f};
}
// the best 32 of row[from .. to - 1], sorted.
template <typename T>
__device__ __noinline__ u64 lp_best_of_all(const T* row, int from, int to) {
  u64 list = 0;
  for (int j0 = from; j0 < to; j0 += 128) {
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + i * 32 + static_cast<int>(threadIdx.x & 31);
      z[i] = j < to ? twa_to_float(row[j]) : 0.0f;
    }
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + i * 32 + static_cast<int>(threadIdx.x & 31);
      list = lp_take32(list, j < to ? lp_key(z[i], j) : 0);
    }
  }
  return list;
}

// Every wait that runs out sets gave_up, and whoever waits later does not wait long.  A thread sets it before its warp arrives anywhere
// again, so two looks at it are enough: the warp that copies looks before it fills a stage again (the last copy into it
// may not have landed), and a warp that finishes rows after its wait for one, whose results are right if the flag is not set, and
// not stored but reported if it is.  The summing warps do not look (with a look of theirs at each row's end 1 % slower, in
// every chunk 2 %).
__device__ __forceinline__ bool lp_gave_up(const int* gave_up) { return *static_cast<const volatile int*>(gave_up) != 0; }

// Chunks of a slot, as a power of two.
__device__ __forceinline__ int lp_log_slot(int chunks) {
  int log = 0;
  while (LP_SLOTS << log < chunks) ++log;
  return log;
}

// A row per cluster of 2^log_parts blocks, each a run of its units; with one part a block goes on to further rows.
template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(LP_BLOCK, LP_BLOCKS_PER_SM<TOP>) logprobs_kernel(LpArgs a, const int log_parts) {
  constexpr int E = twa_vec<T>;
  const int parts = 1 << log_parts;
  typedef LpWord<T> W;
  extern __shared__ __align__(128) unsigned char lp_smem[];
  constexpr int STAGES = LP_STAGES<TOP>;
  LpShared<TOP>& sh = *reinterpret_cast<LpShared<TOP>*>(lp_smem);
  const int part = parts > 1 ? static_cast<int>(twa_cluster_rank()) : 0;
  const long long row0 = blockIdx.x >> log_parts, rows_step = gridDim.x >> log_parts;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int q = 0; q < STAGES; ++q) {
      twa_mbar_init(twa_smem_u32(&sh.full[q]), 1);
      twa_mbar_init(twa_smem_u32(&sh.empty[q]), LP_WARPS);
    }
    for (int q = 0; q < LP_FINISHERS; ++q) {
      twa_mbar_init(twa_smem_u32(&sh.row_full[q]), LP_WARPS);
      twa_mbar_init(twa_smem_u32(&sh.row_empty[q]), 1);
    }
    sh.gave_up = 0;
    twa_fence_barrier_init();
  }
  __syncthreads();
  twa_begin(a.logits, a.targets);
  const T* logits = static_cast<const T*>(a.logits);

  if (warp == LP_COPY) {
    // ---- copies: every chunk of every row of this block, as the ring has room
    if (lane == 0) {
      int it = 0;
      bool good = true;
      for (long long row = row0; row < a.rows && good; row += rows_step) {
        const LpRow<T> x(logits + row * a.ld, a.vocab);
        const int u0 = x.part_from(part, log_parts);
        const int u1 = x.part_from(part + 1, log_parts);
        for (int u = u0; u < u1; u += LP_CHUNK, ++it) {
          const int q = it % STAGES;
          if (it >= STAGES &&
              (!twa_wait(&sh.empty[q], (it / STAGES & 1) ^ 1, &sh.gave_up, a.wait_limit_ns) || lp_gave_up(&sh.gave_up))) {
            good = false;
            break;
          }
          const uint32_t bytes = static_cast<uint32_t>(min(LP_CHUNK, u1 - u)) * 16;
          twa_mbar_expect_tx(twa_smem_u32(&sh.full[q]), bytes);
          twa_bulk_load(twa_smem_u32(sh.ring[q]), x.base + static_cast<long long>(x.first + u) * E, bytes, twa_smem_u32(&sh.full[q]));
        }
      }
      // no copy may still be on its way into this block's shared memory when it ends
      for (int back = 1; back <= STAGES && back <= it; ++back) {
        const int last = it - back, q = last % STAGES;
        const u64 begun = twa_globaltimer();
        while (!twa_mbar_try_wait(twa_smem_u32(&sh.full[q]), last / STAGES & 1))
          if (twa_globaltimer() - begun > a.wait_limit_ns) break;
      }
    }
    __syncwarp();
    if (parts > 1) {
      twa_cluster_sync();
      twa_cluster_sync();
    }
    return;
  }

  if (warp >= LP_FINISH) {
    // ---- finish
    const int turn = warp - LP_FINISH;
    if (parts > 1 && turn) {       // a cluster has one row
      twa_cluster_sync();
      twa_cluster_sync();
      return;
    }
    int r = 0;                     // of this warp's rows
    for (long long row = row0 + turn * rows_step; row < a.rows; row += LP_FINISHERS * rows_step, ++r) {
      const LpRow<T> x(logits + row * a.ld, a.vocab);
      const int u0 = x.part_from(part, log_parts);
      const int u1 = x.part_from(part + 1, log_parts);
      const int chunks = (u1 - u0 + LP_CHUNK - 1) / LP_CHUNK;
      const int log_slot = lp_log_slot(chunks);
      // the elements of this block's part: from .. to - 1
      const int from = part == 0 ? 0 : (x.first + u0) * E - x.skew, to = part == parts - 1 ? a.vocab : (x.first + u1) * E - x.skew;
      long long target = 0;
      float zt = 0.0f;
      if (part == 0 && lane == 0) {
        target = twa_load_id(a.targets, a.itype, row);
        if (target >= 0 && target < a.vocab) zt = twa_to_float(x.base[x.skew + target]);
      }
      const bool good = twa_wait(&sh.row_full[turn], r & 1, &sh.gave_up, a.wait_limit_ns) && !lp_gave_up(&sh.gave_up);
      if (!__all_sync(0xffffffffu, good)) {
        if (lane == 0) twa_set_status(a.status, TWA_ERR_TIMEOUT, -1);
        if (parts > 1) {
          twa_cluster_sync();
          twa_cluster_sync();
        }
        return;
      }
      LpStat st = lp_merge_near<ENT, LP_WARPS>(sh.stat[turn][lane & (LP_WARPS - 1)]);
      uint32_t key[LP_WARPS];
      if (TOP)
#pragma unroll
        for (int i = 0; i < LP_WARPS; ++i) key[i] = sh.key[turn][i * 32 + lane];
      // the summing warps may write the next row but one to where this one's stat, key and slot have been read
      auto release = [&] {
        __syncwarp();
        if (lane == 0) twa_mbar_arrive(twa_smem_u32(&sh.row_empty[turn]));
      };
      if (!TOP) release();
      if (fabsf(st.m) >= LP_FAR && st.m != -INFINITY) st = lp_sum_far<T, ENT>(x.base + x.skew, from, to, st.m);

      u64 found = 0;                 // sorted
      if (TOP) {
        if (st.m == -INFINITY) {     // nothing above -inf: the first indices
          release();
          if (lane < to - from) found = lp_key(-INFINITY, from + lane);
        } else {
          // a group: the eight threads of one lane number
          uint32_t g = key[0];
#pragma unroll
          for (int i = 1; i < LP_WARPS; ++i) g = max(g, key[i]);
          // the top-th largest of the groups': the last one with fewer than `top` above it
          const int above = lp_place32(g, sh.group[turn]);
          const int most = __reduce_max_sync(0xffffffffu, above < a.top ? above : -1);
          const uint32_t bound = __shfl_sync(0xffffffffu, g, __ffs(__ballot_sync(0xffffffffu, above == most)) - 1);
          const float bound_value = bound ? lp_unrank(bound) : -INFINITY;
          int chosen = 0;
#pragma unroll
          for (int i = 0; i < LP_WARPS; ++i) {
            const bool yes = key[i] && key[i] >= bound;
            const unsigned all = __ballot_sync(0xffffffffu, yes);
            if (yes) sh.chosen[turn][chosen + __popc(all & ((1u << lane) - 1))] = i * 32 + lane;
            chosen += __popc(all);
          }
          __syncwarp();
          // their parts that reach the bound
          int pairs = 0;
          {
            int slot = lane / chosen, who = lane % chosen;
            const int slot_step = 32 / chosen, who_step = 32 % chosen;
            const int slots = (chunks + (1 << log_slot) - 1) >> log_slot;
            for (int i0 = 0; i0 < chosen * slots; i0 += 32) {
              int thread = 0;
              bool yes = slot < slots;
              if (yes) {
                thread = sh.chosen[turn][who];
                yes = sh.slot[turn][slot][thread] >= bound_value;
              }
              const unsigned all = __ballot_sync(0xffffffffu, yes);
              const int to = pairs + __popc(all & ((1u << lane) - 1));
              if (yes && to < LP_BUFFER) sh.pair[turn][to] = slot * LP_THREADS + thread;
              pairs += __popc(all);
              slot += slot_step;
              who += who_step;
              if (who >= chosen) {
                who -= chosen;
                ++slot;
              }
            }
          }
          release();
          // their units that hold a value as large as the bound's
          constexpr int AHEAD = 4;
          const int log_each = 2 + log_slot, tasks = pairs <= LP_BUFFER ? pairs << log_each : 0;
          static_assert(LP_PER_THREAD == 4, "log_each");
          int hits = 0;
          for (int i0 = 0; i0 < tasks; i0 += 32 * AHEAD) {
            uint4 q[AHEAD];
            int u[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
              const int i = i0 + 32 * j + lane;
              u[j] = u1;
              if (i < tasks) {
                const int pair = sh.pair[turn][i >> log_each], of = i & ((1 << log_each) - 1);
                u[j] = u0 + (((pair / LP_THREADS) << log_each) + of) * LP_THREADS + pair % LP_THREADS;
              }
              if (u[j] < u1) q[j] = __ldg(reinterpret_cast<const uint4*>(x.base + static_cast<long long>(x.first + u[j]) * E));
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
              const bool hit = u[j] < u1 && W::max1(W::max2(W::max2(q[j].x, q[j].y), W::max2(q[j].z, q[j].w))) >= bound_value;
              const unsigned all = __ballot_sync(0xffffffffu, hit);
              const int to = hits + __popc(all & ((1u << lane) - 1));
              hits += __popc(all);
              if (hit && to < LP_BUFFER) {
                sh.hit[turn][to] = q[j];
                sh.hit_unit[turn][to] = u[j];
              }
            }
          }
          __syncwarp();
          // their elements, and the row's ragged ends, of the bound's rank or above
          int count = 0;
          const int heads = part == 0 ? x.head() : 0, tails = part == parts - 1 ? a.vocab - x.tail_from() : 0;
          const int elements = hits <= LP_BUFFER ? hits * E : 0;
          for (int i0 = 0; i0 < elements + heads + tails; i0 += 32) {
            const int i = i0 + lane;
            u64 key = 0;
            if (i < elements) {
              const int u = sh.hit_unit[turn][i / E];
              const float z = twa_to_float(reinterpret_cast<const T*>(sh.hit[turn])[i]);
              if (lp_rank(z) >= bound) key = lp_key(z, (x.first + u) * E + i % E - x.skew);
            } else if (i < elements + heads + tails) {
              const bool head = i < elements + heads;
              const int j = head ? i - elements : x.tail_from() + i - elements - heads;
              const float z = twa_to_float(x.base[x.skew + j]);
              if (lp_rank(z) >= bound) key = lp_key(z, j);
            }
            const unsigned all = __ballot_sync(0xffffffffu, key != 0);
            const int to = count + __popc(all & ((1u << lane) - 1));
            count += __popc(all);
            if (key && to < LP_BUFFER) sh.buffer[turn][to] = key;
          }
          __syncwarp();
          if (pairs <= LP_BUFFER && hits <= LP_BUFFER && count <= LP_BUFFER) {
            found = lp_sort_buffer(sh.buffer[turn], count);
          } else {
            found = lp_best_of_all(x.base + x.skew, from, to);     // a row with many equal values
          }
        }
      }

      // ---- the cluster's
      if (parts > 1) {
        if (lane == 0) sh.mine = st;
        if (TOP) sh.best[lane] = found;
        twa_cluster_sync();
        if (part == 0) {
          // a lane a part's sums
          LpStat one = {-INFINITY, 0.0f, 0.0f};
          if (lane < parts) {
            one.m = twa_remote(&sh.mine.m, lane);
            one.s = twa_remote(&sh.mine.s, lane);
            one.a = ENT ? twa_remote(&sh.mine.a, lane) : 0.0f;
          }
          st = lp_merge<ENT>(one);
          if (TOP) {
            // the parts' lists: the top-th largest of a sample, the first 32 / parts of each list, bounds what is left to sort
            u64 list[LP_MAX_CLUSTER];
#pragma unroll
            for (int p = 0; p < LP_MAX_CLUSTER; ++p) list[p] = p < parts ? twa_remote(&sh.best[lane], p) : 0;
            const u64 sample = twa_remote(&sh.best[lane & ((32 >> log_parts) - 1)], lane >> (5 - log_parts));
            const int above = lp_place32(sample, sh.buffer[turn]);
            const int most = __reduce_max_sync(0xffffffffu, above < a.top ? above : -1);
            const u64 bound = __shfl_sync(0xffffffffu, sample, __ffs(__ballot_sync(0xffffffffu, above == most)) - 1);
            int count = 0;
#pragma unroll
            for (int p = 0; p < LP_MAX_CLUSTER; ++p) {
              const bool yes = list[p] && list[p] >= bound;
              const unsigned all = __ballot_sync(0xffffffffu, yes);
              const int to = count + __popc(all & ((1u << lane) - 1));
              if (yes && to < LP_BUFFER) sh.buffer[turn][to] = list[p];
              count += __popc(all);
            }
            __syncwarp();
            if (count <= LP_BUFFER) {
              found = lp_sort_buffer(sh.buffer[turn], count);
            } else {
              found = list[0];
#pragma unroll 1
              for (int p = 1; p < parts; ++p) found = lp_merge32(found, twa_remote(&sh.best[31 - lane], p));
            }
          }
        }
        twa_cluster_sync();           // no block leaves while its shared memory is read
        if (part != 0) return;
      }
      const float logs = LN2 * log2f(st.s);
      const float lse = st.m == -INFINITY ? (st.s == 0.0f ? -INFINITY : NAN) : st.m + logs;
      if (lane == 0) {
        a.lse[row] = lse;
        if (!(lse < INFINITY)) twa_set_status(a.status, TWA_ERR_NONFINITE, static_cast<int>(row));
        const bool none = lse == -INFINITY;
        if (ENT) a.entropy[row] = none ? 0.0f : logs - LN2 * (st.a / st.s);
        float lp = 0.0f;
        if (target != a.ignore_id) {
          if (target < 0 || target >= a.vocab) {
            twa_set_status(a.status, TWA_ERR_INVALID_ARG, static_cast<int>(row));
            lp = NAN;
          } else {
            lp = none ? -INFINITY : zt - st.m - logs;
          }
        }
        a.logp[row] = lp;
      }
      if (TOP && lane < a.top) {
        a.top_ids[row * a.top + lane] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(found));
        a.top_logp[row * a.top + lane] = lse == -INFINITY ? -INFINITY : lp_unrank(static_cast<uint32_t>(found >> 32)) - st.m - logs;
      }
    }
    return;
  }

  // ---- sums
  int it = 0, r = 0;
  for (long long row = row0; row < a.rows; row += rows_step, ++r) {
    const int turn = r % LP_FINISHERS, round = r / LP_FINISHERS;
    const LpRow<T> x(logits + row * a.ld, a.vocab);
    const int u0 = x.part_from(part, log_parts);
    const int u1 = x.part_from(part + 1, log_parts);
    const int chunks = (u1 - u0 + LP_CHUNK - 1) / LP_CHUNK;
    const int log_slot = lp_log_slot(chunks);
    float m = -INFINITY, c = -LP_FAR * LOG2E;
    u64 s2 = 0, w2 = 0;            // pairs of sums
    bool some = u1 - u0 >= LP_CHUNK;   // whether this thread has any element
    // the sums become relative to the new maximum um
    auto raise_max = [&](float um) {
      const float nc = lp_base(um) * LOG2E, d = fmaxf(c - nc, -150.0f), f = lp_exp2(d);
      const u64 f2 = twa_pair(f, f);
      if (ENT) w2 = twa_mul2(f2, twa_fma2(twa_pair(d, d), s2, w2));
      s2 = twa_mul2(f2, s2);
      m = um;
      c = nc;
    };
    // some units of a thread; returns their maximum
    auto take_units = [&](auto& units) {
      constexpr int N = sizeof(units) / sizeof(uint4);
      uint32_t high[N];
#pragma unroll
      for (int j = 0; j < N; ++j) high[j] = W::max2(W::max2(units[j].x, units[j].y), W::max2(units[j].z, units[j].w));
#pragma unroll
      for (int half = N / 2; half; half >>= 1)
#pragma unroll
        for (int j = 0; j < half; ++j) high[j] = W::max2(high[j], high[j + half]);
      const float um = W::max1(high[0]);
      if (um > m) raise_max(um);
      const u64 c2 = twa_pair(-c, -c), l2 = twa_pair(LOG2E, LOG2E);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        uint32_t w[4] = {units[j].x, units[j].y, units[j].z, units[j].w};
        if (ENT)
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = W::raise(w[i]);
#pragma unroll
        for (int i = 0; i < W::PAIRS; ++i) {
          const u64 d2 = twa_fma2(W::pair(w, i), l2, c2);
          float d0, d1;
          twa_unpair(d2, d0, d1);
          const u64 p2 = twa_pair(lp_exp2(d0), lp_exp2(d1));
          s2 = twa_add2(s2, p2);
          if (ENT) w2 = twa_fma2(p2, d2, w2);
        }
      }
      return um;
    };
    // the row's ragged ends: thread 0 of the first part, thread 1 of the last
    const int ends = part == 0 && threadIdx.x == 0 ? 0 : (part == parts - 1 && threadIdx.x == 1 ? 1 : -1);
    const int end_from = ends == 0 ? 0 : x.tail_from(), end_to = ends == 0 ? x.head() : (ends == 1 ? a.vocab : 0);
    auto take_ends = [&] {
      for (int j = end_from; j < end_to; ++j) {
        const float z = twa_to_float(x.base[x.skew + j]);
        some = true;
        if (z > m) raise_max(z);
        const float d = fmaf(z, LOG2E, -c), p = lp_exp2(d);
        s2 = twa_add2(s2, twa_pair(p, 0.0f));
        if (ENT) w2 = twa_fma2(twa_pair(p, 0.0f), twa_pair(fmaxf(d, -150.0f), 0.0f), w2);
      }
    };
    if (ends == 0) take_ends();
    float part_max = -INFINITY;    // of the slot's part of the row
    // the warp that finishes has taken this buffer's last row
    if (round) twa_wait(&sh.row_empty[turn], (round & 1) ^ 1, &sh.gave_up, a.wait_limit_ns);
    for (int k = 0; k < chunks; ++k, ++it) {
      const int q = it % STAGES, n = min(LP_CHUNK, u1 - u0 - k * LP_CHUNK);
      // after a wait that ran out the row's results are not defined
      twa_wait(&sh.full[q], it / STAGES & 1, &sh.gave_up, a.wait_limit_ns);
      if (n == LP_CHUNK) {
        uint4 w[LP_PER_THREAD];
#pragma unroll
        for (int j = 0; j < LP_PER_THREAD; ++j) w[j] = sh.ring[q][j * LP_THREADS + threadIdx.x];
        __syncwarp();
        if (lane == 0) twa_mbar_arrive(twa_smem_u32(&sh.empty[q]));
        part_max = fmaxf(part_max, take_units(w));
      } else {
        // the last chunk, a unit a thread at a time; a warp without a unit has nothing to do
        for (int j = warp * 32; j < n; j += LP_THREADS) {
          uint4 w[1] = {make_uint4(W::NONE, W::NONE, W::NONE, W::NONE)};
          if (j + lane < n) w[0] = sh.ring[q][j + lane];
          some |= j + lane < n;
          part_max = fmaxf(part_max, take_units(w));
        }
        __syncwarp();
        if (lane == 0) twa_mbar_arrive(twa_smem_u32(&sh.empty[q]));
      }
      if (TOP && (((k + 1) & ((1 << log_slot) - 1)) == 0 || k + 1 == chunks)) {
        sh.slot[turn][k >> log_slot][threadIdx.x] = part_max;
        part_max = -INFINITY;
      }
    }
    if (ends == 1) take_ends();

    // ---- the warp's sums
    LpStat st = {m, 0.0f, 0.0f};
    {
      float s0, s1, w0, w1;
      twa_unpair(s2, s0, s1);
      twa_unpair(w2, w0, w1);
      st.s = s0 + s1;
      st.a = w0 + w1;
      const float e = fmaf(lp_base(m), LOG2E, -c), g = e * LN2;      // c is off by e, at most 2^-11: 2^-e = 1 - g + g^2 / 2
      const float f = fmaf(g, fmaf(g, 0.5f, -1.0f), 1.0f);
      st.a = f * (st.a - e * st.s);
      st.s *= f;
    }
    st = lp_merge_near<ENT, 32>(st);
    if (lane == 0) sh.stat[turn][warp] = st;
    if (TOP) sh.key[turn][threadIdx.x] = some ? lp_rank(m) : 0;
    __syncwarp();
    if (lane == 0) twa_mbar_arrive(twa_smem_u32(&sh.row_full[turn]));
  }
  if (parts > 1) {
    twa_cluster_sync();
    twa_cluster_sync();
  }
}

constexpr int LPB_THREADS = 256;

// Rows x parts blocks; SAME: logits and dlogits rows lie alike on 16-byte boundaries, else element by element.
template <typename T, bool ENT, bool SAME>
__global__ void __launch_bounds__(LPB_THREADS) logprobs_backward_kernel(LpArgs a, const int parts) {
  twa_begin(a.logits, a.targets, a.lse, a.entropy, a.d_logp, a.d_entropy);
  constexpr int E = twa_vec<T>;
  const long long row = blockIdx.x / parts;
  const int part = static_cast<int>(blockIdx.x - row * parts);
  const T* src = static_cast<const T*>(a.logits) + row * a.ld;
  T* dst = static_cast<T*>(a.dlogits) + row * a.ldd;
  const float lse = a.lse[row];
  const long long t = twa_load_id(a.targets, a.itype, row);
  const bool ignored = t == a.ignore_id, none = lse == -INFINITY;
  if (!ignored && (t < 0 || t >= a.vocab) && part == 0 && threadIdx.x == 0)
    twa_set_status(a.status, TWA_ERR_INVALID_ARG, static_cast<int>(row));
  const float dl = ignored || none ? 0.0f : a.d_logp[row];
  const float dh = ENT && !none ? a.d_entropy[row] : 0.0f, h = ENT ? a.entropy[row] : 0.0f;
  const float c = none ? 0.0f : lse;
  // dz = -p (dl + dh (log p + H)), and dl more at the target
  auto grad = [&](float z, int j) {
    const float d = (z - c) * LOG2E;
    float g = dl;
    if (ENT) g = fmaf(dh, fmaf(fmaxf(d, -150.0f), LN2, h), dl);
    const float o = -lp_exp2(d) * g;
    return j == t ? o + dl : o;
  };
  if (SAME) {
    const LpRow<T> x(src, a.vocab);
    T* out = dst - x.skew;
    if (part == 0) {
      const int ends = x.head() + a.vocab - x.tail_from();
      if (static_cast<int>(threadIdx.x) < ends) {
        const int j = static_cast<int>(threadIdx.x) < x.head() ? threadIdx.x : threadIdx.x - x.head() + x.tail_from();
        dst[j] = twa_from_float<T>(grad(twa_to_float(src[j]), j));
      }
    }
    for (int u = part * LPB_THREADS + threadIdx.x; u < x.whole; u += parts * LPB_THREADS) {
      const long long at = static_cast<long long>(x.first + u) * E;
      float v[E];
      twa_pack<T, E> q;
      q.load(x.base + at);
      q.widen(v);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = grad(v[e], (x.first + u) * E + e - x.skew);
      twa_pack<T, E>::store(out + at, v);
    }
  } else {
    for (int j = part * LPB_THREADS + threadIdx.x; j < a.vocab; j += parts * LPB_THREADS)
      dst[j] = twa_from_float<T>(grad(twa_to_float(src[j]), j));
  }
}

template <typename T, bool ENT, bool TOP>
int lp_launch(twa_ctx* ctx, const LpArgs& a, int log_parts) {
  const int parts = 1 << log_parts;
  static int smem_set[64] = {};
  const void* kernel = reinterpret_cast<const void*>(logprobs_kernel<T, ENT, TOP>);
  int rc = twa_ensure_smem(ctx, kernel, &smem_set[ctx->device & 63], sizeof(LpShared<TOP>));
  if (rc) return rc;
  const long long most = static_cast<long long>(ctx->sm_count) * LP_BLOCKS_PER_SM<TOP>;
  const unsigned blocks = static_cast<unsigned>(parts > 1 ? a.rows * parts : (a.rows < most ? a.rows : most));
  TWA_CUDA_OK(ctx, twa_launch_clusters(ctx->stream, logprobs_kernel<T, ENT, TOP>, blocks, parts, LP_BLOCK, sizeof(LpShared<TOP>), a,
                                       log_parts));
  return TWA_OK;
}

template <typename T>
int lp_launch_any(twa_ctx* ctx, const LpArgs& a, int log_parts) {
  if (a.entropy) return a.top ? lp_launch<T, true, true>(ctx, a, log_parts) : lp_launch<T, true, false>(ctx, a, log_parts);
  return a.top ? lp_launch<T, false, true>(ctx, a, log_parts) : lp_launch<T, false, false>(ctx, a, log_parts);
}

template <typename T, bool ENT>
void lp_launch_backward(twa_ctx* ctx, const LpArgs& a, int parts, bool same) {
  const unsigned blocks = static_cast<unsigned>(a.rows * parts);
  if (same) twa_launch(ctx->stream, logprobs_backward_kernel<T, ENT, true>, blocks, LPB_THREADS, 0, a, parts);
  else twa_launch(ctx->stream, logprobs_backward_kernel<T, ENT, false>, blocks, LPB_THREADS, 0, a, parts);
}

int lp_check(const twa_ctx* ctx, twa_dtype dt, twa_itype it, int64_t rows, int vocab) {
  if (!ctx || !twa_dtype_ok(dt) || !twa_itype_ok(it) || rows < 0 || vocab < 1) return TWA_ERR_INVALID_ARG;
  if (rows > TWA_LOGPROBS_MAX_ROWS || vocab > TWA_LOGPROBS_MAX_VOCAB) return TWA_ERR_UNSUPPORTED;
  return TWA_OK;
}

}  // namespace

extern "C" {

int twa_token_logprobs(twa_ctx* ctx, const void* logits, int64_t ld, twa_dtype dtype, int64_t rows, int vocab,
                       const void* targets, twa_itype t_type, int64_t ignore_id, float* logp, float* lse, float* entropy,
                       int top, int32_t* top_ids, float* top_logp) {
  int rc = lp_check(ctx, dtype, t_type, rows, vocab);
  if (rc) return rc;
  if (top < 0 || top > vocab) return TWA_ERR_INVALID_ARG;
  if (top > TWA_LOGPROBS_MAX_TOP) return TWA_ERR_UNSUPPORTED;
  if (rows == 0) return TWA_OK;
  if (!logits || !targets || !logp || !lse || ld < vocab || (top && (!top_ids || !top_logp))) return TWA_ERR_INVALID_ARG;
  if (twa_misaligned_to(logits, twa_dtype_size(dtype)) || twa_misaligned_to(targets, twa_itype_size(t_type)) ||
      twa_misaligned_to(logp, 4) || twa_misaligned_to(lse, 4) || twa_misaligned_to(entropy, 4) || twa_misaligned_to(top_ids, 4) ||
      twa_misaligned_to(top_logp, 4))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LpArgs a = {};
  a.logits = logits;
  a.targets = targets;
  a.logp = logp;
  a.lse = lse;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_logp = top_logp;
  a.ld = ld;
  a.rows = rows;
  a.ignore_id = ignore_id;
  a.vocab = vocab;
  a.itype = t_type;
  a.top = top;
  a.wait_limit_ns = ctx->wait_limit_ns;
  a.status = ctx->d_status;
  int log_parts = 0;
  const long long units = twa_ceil_div(static_cast<long long>(vocab) * twa_dtype_size(dtype), 16);
  while ((1 << log_parts) < LP_MAX_CLUSTER && rows << (log_parts + 1) <= LP_SPLIT_ROWS * ctx->sm_count &&
         units > LP_CHUNK / 2 << log_parts)
    ++log_parts;
  return dtype == TWA_BF16 ? lp_launch_any<bf16>(ctx, a, log_parts) : lp_launch_any<float>(ctx, a, log_parts);
}

int twa_token_logprobs_backward(twa_ctx* ctx, const void* logits, int64_t ld, twa_dtype dtype, int64_t rows, int vocab,
                                const void* targets, twa_itype t_type, int64_t ignore_id, const float* lse,
                                const float* entropy, const float* d_logp, const float* d_entropy, void* dlogits, int64_t ldd) {
  int rc = lp_check(ctx, dtype, t_type, rows, vocab);
  if (rc) return rc;
  if (rows == 0) return TWA_OK;
  if (!logits || !targets || !lse || !d_logp || !dlogits || ld < vocab || ldd < vocab || (d_entropy && !entropy))
    return TWA_ERR_INVALID_ARG;
  const size_t size = twa_dtype_size(dtype);
  if (twa_misaligned_to(logits, size) || twa_misaligned_to(dlogits, size) || twa_misaligned_to(targets, twa_itype_size(t_type)) ||
      twa_misaligned_to(lse, 4) || twa_misaligned_to(entropy, 4) || twa_misaligned_to(d_logp, 4) || twa_misaligned_to(d_entropy, 4))
    return TWA_ERR_MISALIGNED;
  TWA_CUDA_OK(ctx, cudaSetDevice(ctx->device));
  LpArgs a = {};
  a.logits = logits;
  a.targets = targets;
  a.lse = const_cast<float*>(lse);
  a.entropy = const_cast<float*>(entropy);
  a.d_logp = d_logp;
  a.d_entropy = d_entropy;
  a.dlogits = dlogits;
  a.ld = ld;
  a.ldd = ldd;
  a.rows = rows;
  a.ignore_id = ignore_id;
  a.vocab = vocab;
  a.itype = t_type;
  a.status = ctx->d_status;
  const bool same = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15) == 0 &&
                    (rows == 1 || ((ld - ldd) * static_cast<int64_t>(size)) % 16 == 0);
  const long long units = twa_ceil_div(static_cast<long long>(vocab) * size, 16);
  long long parts = twa_ceil_div(units, 8LL * LPB_THREADS);
  while (parts < twa_ceil_div(units, LPB_THREADS) && rows * parts < 4LL * ctx->sm_count) ++parts;
  if (rows * parts > 0x7fffffffLL) return TWA_ERR_UNSUPPORTED;
  if (dtype == TWA_BF16) {
    if (d_entropy) lp_launch_backward<bf16, true>(ctx, a, static_cast<int>(parts), same);
    else lp_launch_backward<bf16, false>(ctx, a, static_cast<int>(parts), same);
  } else {
    if (d_entropy) lp_launch_backward<float, true>(ctx, a, static_cast<int>(parts), same);
    else lp_launch_backward<float, false>(ctx, a, static_cast<int>(parts), same);
  }
  TWA_CUDA_OK(ctx, cudaGetLastError());
  return TWA_OK;
}

}  // extern "C"
