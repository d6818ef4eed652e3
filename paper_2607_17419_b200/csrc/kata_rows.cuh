// Entries of a row, a few at a time: as they lie in memory, as fp32, and back (rounded to nearest even).
#pragma once

#include "kata_common.cuh"

namespace kata {

template <int BYTES> struct RawBytes;
template <> struct RawBytes<16> { typedef uint4 type; };
template <> struct RawBytes<8> { typedef uint2 type; };
template <> struct RawBytes<4> { typedef uint32_t type; };
template <> struct RawBytes<2> { typedef uint16_t type; };

__device__ __forceinline__ void words(const uint4& r, uint32_t (&u)[4]) { u[0] = r.x; u[1] = r.y; u[2] = r.z; u[3] = r.w; }
__device__ __forceinline__ void words(const uint2& r, uint32_t (&u)[2]) { u[0] = r.x; u[1] = r.y; }
__device__ __forceinline__ void words(const uint32_t& r, uint32_t (&u)[1]) { u[0] = r; }
__device__ __forceinline__ void from_words(const uint32_t (&u)[4], uint4& r) { r = make_uint4(u[0], u[1], u[2], u[3]); }
__device__ __forceinline__ void from_words(const uint32_t (&u)[2], uint2& r) { r = make_uint2(u[0], u[1]); }
__device__ __forceinline__ void from_words(const uint32_t (&u)[1], uint32_t& r) { r = u[0]; }

// N entries of type T, loaded and stored in one access (aligned to their size).
template <typename T, int N> struct Entries {
  typedef typename RawBytes<sizeof(T) * N>::type Raw;
  Raw raw;
  __device__ __forceinline__ void load(const void* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void store(void* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ void zero() { raw = Raw{}; }
  // (bf16 two at a time: an entry alone is converted on the pipe of the transcendental functions, an eighth as fast)
  __device__ __forceinline__ void get(float (&x)[N]) const {
    if constexpr (sizeof(T) == 2 && N % 2 == 0) {
      uint32_t u[N / 2];
      words(raw, u);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      }
    } else if constexpr (sizeof(T) == 4) {
      uint32_t u[N];
      words(raw, u);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = __uint_as_float(u[i]);
    } else {
      x[0] = __uint_as_float((uint32_t)raw << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
    if constexpr (sizeof(T) == 2 && N % 2 == 0) {
      uint32_t u[N / 2];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&v);
      }
      from_words(u, raw);
    } else if constexpr (sizeof(T) == 4) {
      uint32_t u[N];
#pragma unroll
      for (int i = 0; i < N; ++i) u[i] = __float_as_uint(x[i]);
      from_words(u, raw);
    } else {
      raw = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
    }
  }
};

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(*reinterpret_cast<unsigned long long*>(&d))
      : "l"(*reinterpret_cast<const unsigned long long*>(&a)), "l"(*reinterpret_cast<const unsigned long long*>(&b)),
        "l"(*reinterpret_cast<const unsigned long long*>(&c)));
  return d;
}

__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<unsigned long long*>(&d))
      : "l"(*reinterpret_cast<const unsigned long long*>(&a)), "l"(*reinterpret_cast<const unsigned long long*>(&b)));
  return d;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<unsigned long long*>(&d))
      : "l"(*reinterpret_cast<const unsigned long long*>(&a)), "l"(*reinterpret_cast<const unsigned long long*>(&b)));
  return d;
}

// Launches with programmatic stream serialisation: the kernel may become resident before the one ahead of it in the stream has
// ended, and waits for it (cudaGridDependencySynchronize) before it touches memory.  It lets the kernel behind become resident
// before it has waited itself, so a kernel that is launched behind it in this way must not touch memory ahead of its wait either;
// one that has to (the decode step's second kernel) stands behind a kernel that waits first and lets it start then.
// early = false: it starts when that kernel has ended.
template <typename... P, typename... A>
inline void launch_when(bool early, LaunchCtx& ctx, void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = ctx.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  if (ctx.status != KATA_OK) return;
  if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) != cudaSuccess) {
    cudaGetLastError();
    ctx.status = KATA_ERR_CUDA;
    return;
  }
  ++ctx.launches;
}

template <typename... P, typename... A>
inline void launch_after(LaunchCtx& ctx, void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, A&&... args) {
  launch_when(true, ctx, kernel, grid, block, smem, args...);
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
