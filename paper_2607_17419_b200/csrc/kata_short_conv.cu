// Short causal convolution of every channel along the tokens, and its backward:
//   z_t = bias + sum_{j < W} w[j] x_{t - W + 1 + j},  y_t = z_t or z_t sigmoid(z_t)
//   g_t = dy_t (act'(z_t)),  dx_t = sum_j w[W - 1 - j] g_{t + j},  dw[j] = sum_t g_t x_{t - W + 1 + j},  dbias = sum_t g_t
// HBM-bound: x in and y out (backward: x and dy in, dx out).  A thread walks a segment of the tokens of a few neighbouring channels
// with the last W - 1 inputs in registers, so an input is loaded once but for the W - 1 before a segment; neighbouring threads hold
// neighbouring channels.  The backward recomputes z, and a segment looks W - 1 tokens beyond its end for the gradients that its
// inputs are taps of.  Sums over tokens: registers, then the segments of a block, then the blocks, each in a fixed order.
#include "kata_rows.cuh"

namespace kata {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;              // tokens in flight per thread

// z sigmoid(z) and its derivative.  bf16: the fast exponential and division (2^-21 relative, the result is rounded to 2^-9).
template <typename T> __device__ __forceinline__ float sigmoid_of(float z) {
  if (sizeof(T) == 2) return __fdividef(1.f, 1.f + __expf(-z));       // (1 / (1 + e^-z) is 0 for z below -88, where e^-z is inf)
  return 1.f / (1.f + expf(-z));
}

struct Place {
  int b, seg, c;                       // sequence, segment, first channel
  bool on;
};
// Blocks of tx channel groups x ty segments; the blocks of a row of segments lie side by side.
__device__ __forceinline__ Place place(int groups, int vec, int col_blocks, int segs, long long seg_rows) {
  const int tx = threadIdx.x, ty = threadIdx.y;
  const unsigned cb = blockIdx.x % (unsigned)col_blocks, rb = blockIdx.x / (unsigned)col_blocks;
  const long long row = (long long)rb * blockDim.y + ty;
  const int g = (int)(cb * blockDim.x) + tx;
  Place p;
  p.on = g < groups && row < seg_rows;
  p.b = p.on ? (int)(row / segs) : 0;
  p.seg = p.on ? (int)(row - (long long)p.b * segs) : 0;
  p.c = p.on ? g * vec : 0;
  return p;
}

template <typename T, int W, int VEC>
__device__ __forceinline__ void load_taps(const ShortConv& a, int c, float (&w)[W][VEC], float (&bias)[VEC]) {
  const T* wt = static_cast<const T*>(a.weight) + (size_t)c * W;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = to_f32<T>(wt[i * W + j]);
    bias[i] = a.bias != nullptr ? to_f32<T>(static_cast<const T*>(a.bias)[c + i]) : 0.f;
  }
}

template <typename T, int W, int VEC>
__global__ void __launch_bounds__(kThreads) short_conv_kernel(const __grid_constant__ ShortConv a, int groups, int col_blocks, int segs,
                                                              int seg_tokens) {
  wait_for_kernels_ahead();
  const Place p = place(groups, VEC, col_blocks, segs, (long long)a.B * segs);
  if (!p.on) return;
  const int len = sequence_length(a.lengths, p.b, a.T);
  const T* x = reinterpret_cast<const T*>(a.x.p) + (long long)p.b * a.x.s0 + p.c;
  T* y = reinterpret_cast<T*>(a.out.p) + (long long)p.b * a.out.s0 + p.c;
  float w[W][VEC], bias[VEC], win[W - 1][VEC];
  load_taps<T, W, VEC>(a, p.c, w, bias);
  const int t0 = p.seg * seg_tokens, t1 = min(t0 + seg_tokens, a.T);
  const size_t state = ((size_t)p.b * a.D + p.c) * (W - 1);
  if (p.seg == 0) {
    // the inputs before the first token, and those that the next call finds there (the same thread reads and writes a state)
    const T* s0 = static_cast<const T*>(a.s_init);
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) win[j][i] = s0 != nullptr ? to_f32<T>(s0[state + i * (W - 1) + j]) : 0.f;
    if (a.s_final != nullptr) {
      T* s1 = static_cast<T*>(a.s_final);
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        const int t = len - (W - 1) + j;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float v = 0.f;
          if (t >= 0) v = to_f32<T>(x[(long long)t * a.x.s1 + i]);
          else {
#pragma unroll
            for (int o = 0; o < W - 1; ++o)
              if (o == t + W - 1) v = win[o][i];
          }
          s1[state + i * (W - 1) + j] = from_f32<T>(v);
        }
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int t = t0 - (W - 1) + j;
      Entries<T, VEC> e;
      e.zero();
      if (t < len) e.load(x + (long long)t * a.x.s1);
      e.get(win[j]);
    }
  }
  for (int t = t0; t < t1; t += kAhead) {
    Entries<T, VEC> in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      in[u].zero();
      if (t + u < min(t1, len)) in[u].load(x + (long long)(t + u) * a.x.s1);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float now[VEC], z[VEC];
      in[u].get(now);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        z[i] = bias[i];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) z[i] = fmaf(w[j][i], win[j][i], z[i]);
        z[i] = fmaf(w[W - 1][i], now[i], z[i]);
        if (a.silu) z[i] *= sigmoid_of<T>(z[i]);
        if (t + u >= len) z[i] = 0.f;
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) win[j][i] = win[j + 1][i];
        win[W - 2][i] = now[i];
      }
      if (t + u < t1) {
        Entries<T, VEC> o;
        o.set(z);
        o.store(y + (long long)(t + u) * a.out.s1);
      }
    }
  }
}

// part: [blocks of segments][W + 1][D], or null where no sum is wanted
template <typename T, int W, int VEC>
__global__ void __launch_bounds__(kThreads) short_conv_bwd_kernel(const __grid_constant__ ShortConv a, int groups, int col_blocks, int segs,
                                                                  int seg_tokens, float* __restrict__ part) {
  extern __shared__ float red[];       // [ty][W + 1][tx * VEC]
  wait_for_kernels_ahead();
  const Place p = place(groups, VEC, col_blocks, segs, (long long)a.B * segs);
  float dw[W + 1][VEC];
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[j][i] = 0.f;
  if (p.on) {
    const int len = sequence_length(a.lengths, p.b, a.T);
    const T* x = reinterpret_cast<const T*>(a.x.p) + (long long)p.b * a.x.s0 + p.c;
    const T* dy = reinterpret_cast<const T*>(a.dout.p) + (long long)p.b * a.dout.s0 + p.c;
    T* dx = reinterpret_cast<T*>(a.dx.p) + (long long)p.b * a.dx.s0 + p.c;
    float w[W][VEC], bias[VEC], win[W - 1][VEC], gw[W - 1][VEC];
    load_taps<T, W, VEC>(a, p.c, w, bias);
    const int t0 = p.seg * seg_tokens, t1 = min(t0 + seg_tokens, a.T);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int t = t0 - (W - 1) + j;
      Entries<T, VEC> e;
      e.zero();
      if (t >= 0 && t < len) e.load(x + (long long)t * a.x.s1);
      e.get(win[j]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) gw[j][i] = 0.f;
    }
    for (int t = t0; t < t1 + W - 1; t += kAhead) {
      Entries<T, VEC> in[kAhead], gin[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        in[u].zero();
        gin[u].zero();
        if (t + u < min(t1 + W - 1, len)) {
          in[u].load(x + (long long)(t + u) * a.x.s1);
          gin[u].load(dy + (long long)(t + u) * a.dout.s1);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float now[VEC], g[VEC], out[VEC];
        in[u].get(now);
        gin[u].get(g);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (a.silu) {
            float z = bias[i];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) z = fmaf(w[j][i], win[j][i], z);
            z = fmaf(w[W - 1][i], now[i], z);
            const float sig = sigmoid_of<T>(z);
            g[i] *= sig * fmaf(z, 1.f - sig, 1.f);
          }
          if (t + u >= len) g[i] = 0.f;
          // the input W - 1 tokens back has met all its taps
          out[i] = w[0][i] * g[i];
#pragma unroll
          for (int j = 0; j < W - 1; ++j) out[i] = fmaf(w[W - 1 - j][i], gw[j][i], out[i]);
          const float own = t + u < t1 ? g[i] : 0.f;
#pragma unroll
          for (int j = 0; j < W - 1; ++j) dw[j][i] = fmaf(own, win[j][i], dw[j][i]);
          dw[W - 1][i] = fmaf(own, now[i], dw[W - 1][i]);
          dw[W][i] += own;
#pragma unroll
          for (int j = 0; j + 1 < W - 1; ++j) {
            win[j][i] = win[j + 1][i];
            gw[j][i] = gw[j + 1][i];
          }
          win[W - 2][i] = now[i];
          gw[W - 2][i] = g[i];
        }
        const int at = t + u - (W - 1);
        if (at >= t0 && at < t1) {
          if (at >= len)
#pragma unroll
            for (int i = 0; i < VEC; ++i) out[i] = 0.f;
          Entries<T, VEC> o;
          o.set(out);
          o.store(dx + (long long)at * a.dx.s1);
        }
      }
    }
  }
  if (part == nullptr) return;
  const int cols = blockDim.x * VEC;
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) red[((size_t)threadIdx.y * (W + 1) + j) * cols + threadIdx.x * VEC + i] = dw[j][i];
  __syncthreads();
  const unsigned cb = blockIdx.x % (unsigned)col_blocks, rb = blockIdx.x / (unsigned)col_blocks;
  for (int e = threadIdx.y * blockDim.x + threadIdx.x; e < (W + 1) * cols; e += blockDim.x * blockDim.y) {
    float sum = 0.f;
    for (int y = 0; y < (int)blockDim.y; ++y) sum += red[(size_t)y * (W + 1) * cols + e];
    const int j = e / cols, c = (int)cb * cols + e % cols;
    if (c < a.D) part[((size_t)rb * (W + 1) + j) * a.D + c] = sum;
  }
}

// dweight[c][j] and dbias[c]: the blocks' sums added in order, eight runs of them side by side.
__global__ void __launch_bounds__(256) short_conv_sum_kernel(const float* __restrict__ part, int blocks, int W, int D,
                                                             float* __restrict__ dweight, float* __restrict__ dbias) {
  __shared__ float red[8][33];
  wait_for_kernels_ahead();
  const int e = blockIdx.x * 32 + threadIdx.x, n = (W + 1) * D;
  float sum = 0.f;
  if (e < n)
    for (int b = threadIdx.y; b < blocks; b += 8) sum += part[(size_t)b * n + e];
  red[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.y != 0 || e >= n) return;
#pragma unroll
  for (int y = 1; y < 8; ++y) sum += red[y][threadIdx.x];
  const int j = e / D, c = e - j * D;
  if (j < W) {
    if (dweight != nullptr) dweight[(size_t)c * W + j] = sum;
  } else if (dbias != nullptr) {
    dbias[c] = sum;
  }
}

struct ConvGrid {
  int groups, col_blocks, segs, seg_tokens;
  dim3 block;
  long long row_blocks;
};
// Segments of 64 tokens; shorter ones (down to 8) while there are fewer threads than the GPU holds.
ConvGrid conv_grid(int B, int T, int D, int vec) {
  ConvGrid g;
  g.groups = (D + vec - 1) / vec;
  int tx = 1;
  while (tx < g.groups && tx < 64) tx *= 2;
  g.block = dim3(tx, kThreads / tx);
  g.col_blocks = (g.groups + tx - 1) / tx;
  g.seg_tokens = 64;
  while (g.seg_tokens > 8 && (double)g.groups * B * ((T + g.seg_tokens - 1) / g.seg_tokens) < kPlanSMs * 1024.0) g.seg_tokens /= 2;
  g.segs = (T + g.seg_tokens - 1) / g.seg_tokens;
  g.row_blocks = ((long long)B * g.segs + g.block.y - 1) / g.block.y;
  return g;
}

bool conv_aligned(const ShortConv& a, const View& v, int bytes) {
  const long long e = a.dtype == KATA_F32 ? 4 : 2;
  return (reinterpret_cast<uintptr_t>(v.p) % bytes) == 0 && (v.s0 * e) % bytes == 0 && (v.s1 * e) % bytes == 0;
}

template <typename T, int W, int VEC> void launch_fwd(const ShortConv& a, LaunchCtx& ctx) {
  const ConvGrid g = conv_grid(a.B, a.T, a.D, VEC);
  launch_after(ctx, short_conv_kernel<T, W, VEC>, dim3((unsigned)(g.row_blocks * g.col_blocks)), g.block, 0, a, g.groups, g.col_blocks, g.segs, g.seg_tokens);
}

template <typename T, int W, int VEC> void launch_bwd(const ShortConv& a, float* ws, LaunchCtx& ctx) {
  const ConvGrid g = conv_grid(a.B, a.T, a.D, VEC);
  const bool sums = a.dweight != nullptr || a.dbias != nullptr;
  const size_t smem = sums ? (size_t)kThreads * VEC * (W + 1) * sizeof(float) : 0;
  launch_after(ctx, short_conv_bwd_kernel<T, W, VEC>, dim3((unsigned)(g.row_blocks * g.col_blocks)), g.block, smem, a, g.groups, g.col_blocks, g.segs,
               g.seg_tokens, sums ? ws : nullptr);
  if (sums)
    launch_after(ctx, short_conv_sum_kernel, dim3(((W + 1) * a.D + 31) / 32), dim3(32, 8), 0, ws, (int)g.row_blocks, W, a.D, a.dweight, a.dbias);
}

constexpr int kBwdVec = 4;             // channels per thread of the backward: eight take 190 registers

template <typename T, int W> void dispatch(const ShortConv& a, bool backward, float* ws, LaunchCtx& ctx) {
  constexpr int V = 16 / sizeof(T);
  if (backward) {
    constexpr int bytes = kBwdVec * sizeof(T);
    if (a.D % kBwdVec == 0 && conv_aligned(a, a.x, bytes) && conv_aligned(a, a.dout, bytes) && conv_aligned(a, a.dx, bytes)) launch_bwd<T, W, kBwdVec>(a, ws, ctx);
    else launch_bwd<T, W, 1>(a, ws, ctx);
  } else if (a.D % V == 0 && conv_aligned(a, a.x, 16) && conv_aligned(a, a.out, 16)) {
    launch_fwd<T, W, V>(a, ctx);
  } else {
    launch_fwd<T, W, 1>(a, ctx);
  }
}

void run(const ShortConv& a, bool backward, float* ws, LaunchCtx& ctx) {
  if (a.dtype == KATA_F32) {
    if (a.W == 2) dispatch<float, 2>(a, backward, ws, ctx);
    else if (a.W == 3) dispatch<float, 3>(a, backward, ws, ctx);
    else dispatch<float, 4>(a, backward, ws, ctx);
  } else {
    if (a.W == 2) dispatch<__nv_bfloat16, 2>(a, backward, ws, ctx);
    else if (a.W == 3) dispatch<__nv_bfloat16, 3>(a, backward, ws, ctx);
    else dispatch<__nv_bfloat16, 4>(a, backward, ws, ctx);
  }
}

}  // namespace

void short_conv_fwd(const ShortConv& a, LaunchCtx& ctx) { run(a, false, nullptr, ctx); }

// (the larger of the two ways to read rows: the scratch does not depend on alignment)
size_t short_conv_bwd_workspace_elems(int B, int T, int D, int W) {
  const long long p = conv_grid(B, T, D, 1).row_blocks, q = conv_grid(B, T, D, kBwdVec).row_blocks;
  return (size_t)(p > q ? p : q) * (W + 1) * D;
}

void short_conv_bwd(const ShortConv& a, float* ws, LaunchCtx& ctx) { run(a, true, ws, ctx); }

}  // namespace kata
