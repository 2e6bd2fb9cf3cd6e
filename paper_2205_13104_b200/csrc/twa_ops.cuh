// Shared by the model-side operators (layer norm, embedding, token log probabilities, clipping): element
// loads and stores of the two types, sums over a warp and a block, argument checks.  sm_100a only.
#pragma once

#include <cuda_bf16.h>
#include <stdio.h>
#include <string.h>

#include "twa_common.cuh"

inline bool twa_dtype_ok(int t) { return t == TWA_F32 || t == TWA_BF16; }
inline bool twa_itype_ok(int t) { return t == TWA_I32 || t == TWA_I64; }
inline size_t twa_dtype_size(int t) { return t == TWA_BF16 ? 2 : 4; }
inline size_t twa_itype_size(int t) { return t == TWA_I64 ? 8 : 4; }
// A pointer to elements of `size` bytes that is not on an element boundary.
inline bool twa_misaligned_to(const void* p, size_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }
inline long long twa_ceil_div(long long a, long long b) { return (a + b - 1) / b; }
inline size_t twa_round256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }

typedef __nv_bfloat16 bf16;

__device__ __forceinline__ float twa_to_float(float v) { return v; }
__device__ __forceinline__ float twa_to_float(bf16 v) { return __bfloat162float(v); }
// One rounding, to nearest even.
template <typename T>
__device__ __forceinline__ T twa_from_float(float v);
template <>
__device__ __forceinline__ float twa_from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 twa_from_float<bf16>(float v) { return __float2bfloat16_rn(v); }

// Element i of an array whose type is known at run time.
__device__ __forceinline__ float twa_load_any(const void* p, int dtype, long long i) {
  return dtype == TWA_BF16 ? __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const unsigned short*>(p) + i)) << 16)
                           : __ldg(static_cast<const float*>(p) + i);
}
__device__ __forceinline__ void twa_store_any(void* p, int dtype, long long i, float v) {
  if (dtype == TWA_BF16) static_cast<bf16*>(p)[i] = twa_from_float<bf16>(v);
  else static_cast<float*>(p)[i] = v;
}
__device__ __forceinline__ long long twa_load_id(const void* p, int itype, long long i) {
  return itype == TWA_I64 ? __ldg(static_cast<const long long*>(p) + i) : static_cast<long long>(__ldg(static_cast<const int*>(p) + i));
}

// E consecutive elements as they lie in memory: E = 1, or 16 bytes (E = 4 float, 8 bfloat16; the address on 16
// bytes).  from() packs values of the type, as widen() gave them.  Loading and widening are apart so that the loads of the next row can be under way while this one is worked on.
template <typename T, int E>
struct twa_pack;
template <>
struct twa_pack<float, 1> {
  float r;
  __device__ __forceinline__ void load(const float* p) { r = __ldg(p); }
  __device__ __forceinline__ void widen(float* v) const { v[0] = r; }
  __device__ __forceinline__ void from(const float* v) { r = v[0]; }
  static __device__ __forceinline__ void store(float* p, const float* v) { *p = v[0]; }
};
template <>
struct twa_pack<bf16, 1> {
  unsigned short r;
  __device__ __forceinline__ void load(const bf16* p) { r = __ldg(reinterpret_cast<const unsigned short*>(p)); }
  __device__ __forceinline__ void widen(float* v) const { v[0] = __uint_as_float(static_cast<uint32_t>(r) << 16); }
  __device__ __forceinline__ void from(const float* v) { r = static_cast<unsigned short>(__float_as_uint(v[0]) >> 16); }
  static __device__ __forceinline__ void store(bf16* p, const float* v) { *p = twa_from_float<bf16>(v[0]); }
};
template <>
struct twa_pack<float, 4> {
  float4 r;
  __device__ __forceinline__ void load(const float* p) { r = __ldg(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void load_shared(const uint4* p) { r = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void widen(float* v) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  __device__ __forceinline__ void from(const float* v) { r = make_float4(v[0], v[1], v[2], v[3]); }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
__device__ __forceinline__ uint32_t twa_bf16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <>
struct twa_pack<bf16, 8> {
  uint4 r;
  __device__ __forceinline__ void load(const bf16* p) { r = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void load_shared(const uint4* p) { r = *p; }
  __device__ __forceinline__ void from(const float* v) {
    r.x = twa_bf16_pair(v[0], v[1]); r.y = twa_bf16_pair(v[2], v[3]);
    r.z = twa_bf16_pair(v[4], v[5]); r.w = twa_bf16_pair(v[6], v[7]);
  }
  __device__ __forceinline__ void widen(float* v) const {
    v[0] = twa_bf16_lo(r.x); v[1] = twa_bf16_hi(r.x); v[2] = twa_bf16_lo(r.y); v[3] = twa_bf16_hi(r.y);
    v[4] = twa_bf16_lo(r.z); v[5] = twa_bf16_hi(r.z); v[6] = twa_bf16_lo(r.w); v[7] = twa_bf16_hi(r.w);
  }
  static __device__ __forceinline__ void store(bf16* p, const float* v) {
    uint4 o;
    o.x = twa_bf16_pair(v[0], v[1]); o.y = twa_bf16_pair(v[2], v[3]);
    o.z = twa_bf16_pair(v[4], v[5]); o.w = twa_bf16_pair(v[6], v[7]);
    *reinterpret_cast<uint4*>(p) = o;
  }
};
template <typename T>
constexpr int twa_vec = 16 / sizeof(T);   // elements of one 16-byte access

__device__ __forceinline__ float twa_warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Pairs of floats: two sums or products an instruction.
typedef unsigned long long twa_f2;
__device__ __forceinline__ twa_f2 twa_pair(float lo, float hi) {
  twa_f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ twa_f2 twa_pair(float both) { return twa_pair(both, both); }
__device__ __forceinline__ void twa_unpair(twa_f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ float twa_pair_sum(twa_f2 v) {
  float lo, hi;
  twa_unpair(v, lo, hi);
  return lo + hi;
}
__device__ __forceinline__ twa_f2 twa_fma2(twa_f2 a, twa_f2 b, twa_f2 c) {
  twa_f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ twa_f2 twa_add2(twa_f2 a, twa_f2 b) {
  twa_f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ twa_f2 twa_mul2(twa_f2 a, twa_f2 b) {
  twa_f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// twa_mbar_wait with a hint to suspend the thread: several warps of a block wait most of the time, and ones that poll
// take issue slots from those that add up.
__device__ __forceinline__ bool twa_wait(unsigned long long* bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
  const uint32_t at = twa_smem_u32(bar);
  unsigned long long begun = 0;
  for (;;) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(at), "r"(parity), "r"(20000u)
        : "memory");
    if (ok) return true;
    if (*abort_flag) return false;
    const unsigned long long now = twa_globaltimer();
    if (!begun) begun = now;
    if (now - begun > limit_ns) {
      *abort_flag = 1;
      return false;
    }
  }
}

// Untiled bulk copy into this block's shared memory: addresses and size in multiples of 16 bytes.
__device__ __forceinline__ void twa_bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// Thread-block clusters: this block's rank, a barrier of all the cluster's threads, and loads and stores of a variable of this
// block's shared memory in the block `rank`.
__device__ __forceinline__ uint32_t twa_cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void twa_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename V>
__device__ __forceinline__ V twa_remote(const V* p, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(twa_smem_u32(p)), "r"(rank));
  V v;
  if constexpr (sizeof(V) == 8) {
    unsigned long long w;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(w) : "r"(at) : "memory");
    v = w;
  } else {
    uint32_t w;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
    memcpy(&v, &w, 4);
  }
  return v;
}

__device__ __forceinline__ void twa_store_remote(unsigned long long* p, uint32_t rank, unsigned long long v) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(twa_smem_u32(p)), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory");
}

// Launches that may begin while the kernel before them in the stream ends (programmatic dependent launch).  A kernel launched
// so first calls twa_begin(pointers it reads ...), which goes on when the kernels before it are complete and their writes
// visible.  The pointers come out of the call as new values, so that no load through them, not even one of data the compiler
// takes for constant, can be moved before it.  No kernel lets the next one begin before its own blocks end: waiting blocks take
// places from the kernel after them (gradient of a layer norm of 16384 x 2048 bfloat16: 63 us if it does, 49 us if not).
template <typename P>
__device__ __forceinline__ void twa_renew(P& pointer) { asm volatile("" : "+l"(pointer) : : "memory"); }
template <typename... P>
__device__ __forceinline__ void twa_begin(P&... pointers) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  (..., twa_renew(pointers));
}

template <typename... Params, typename... Args>
cudaError_t twa_launch_clusters(cudaStream_t stream, void (*kernel)(Params...), dim3 grid, int cluster, int threads, size_t smem,
                                Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
template <typename... Params, typename... Args>
cudaError_t twa_launch(cudaStream_t stream, void (*kernel)(Params...), dim3 grid, int threads, size_t smem, Args... args) {
  return twa_launch_clusters(stream, kernel, grid, 1, threads, smem, args...);
}
