// Entries of a row, a few at a time: as they lie in memory, as fp32, and back (rounded to nearest even).
#pragma once

#include "kata_common.cuh"

namespace kata {

template <int BYTES> struct RawBytes;
template <> struct RawBytes<16> { typedef uint4 type; };
template <> struct RawBytes<8> { typedef uint2 type; };
template <> struct RawBytes<4> { typedef uint32_t type; };
template <> struct RawBytes<2> { typedef uint16_t type; };

// N entries of type T, loaded and stored in one access (aligned to their size).
template <typename T, int N> struct Entries {
  typedef typename RawBytes<sizeof(T) * N>::type Raw;
  Raw raw;
  __device__ __forceinline__ void load(const void* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void load_streaming(const void* p) { raw = __ldcs(reinterpret_cast<const Raw*>(p)); }
  __device__ __forceinline__ void store(void* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ void zero() { raw = Raw{}; }
  __device__ __forceinline__ void get(float (&x)[N]) const {
    const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32<T>(e[i]);
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
    T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = from_f32<T>(x[i]);
  }
};

// Launches with programmatic stream serialisation: the kernel may become resident before the one ahead of it in the stream has
// ended, and waits for it (cudaGridDependencySynchronize) before it touches memory.
template <typename... P, typename... A>
inline void launch_after(LaunchCtx& ctx, void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = ctx.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (ctx.status != KATA_OK) return;
  if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) != cudaSuccess) {
    cudaGetLastError();
    ctx.status = KATA_ERR_CUDA;
    return;
  }
  ++ctx.launches;
}

__device__ __forceinline__ void wait_for_kernels_ahead() {
  cudaTriggerProgrammaticLaunchCompletion();
  cudaGridDependencySynchronize();
}

// Length of sequence b in a padded batch of T tokens.
__device__ __forceinline__ int sequence_length(const int* lengths, int b, int T) {
  return lengths != nullptr ? min(max(lengths[b], 0), T) : T;
}

}  // namespace kata
