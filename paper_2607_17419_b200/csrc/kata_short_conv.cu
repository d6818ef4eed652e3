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
constexpr int kAhead = 2;              // tokens per load step; the next step's are on their way meanwhile

// 1 / (1 + e^-z).  bf16: the approximate exponential and reciprocal (2^-21 relative near 0; for negative z the rounding of the exponent
// comes to |z| 2^-24, 2^-17 at -88; the result is rounded to 2^-8; 0 for z below -88, where e^-z is inf).
template <typename T> __device__ __forceinline__ float sigmoid_of(float z) {
  if (sizeof(T) == 4) return 1.f / (1.f + expf(-z));
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.44269504088896341f * z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
template <typename T> __device__ __forceinline__ float silu_of(float z) {
  return sizeof(T) == 4 ? z / (1.f + expf(-z)) : z * sigmoid_of<T>(z);
}

// The sigmoids of a pair, the products in pairs.
template <typename T> __device__ __forceinline__ float2 sigmoid_pair(float2 z) {
  if (sizeof(T) == 4) return make_float2(sigmoid_of<T>(z.x), sigmoid_of<T>(z.y));
  float2 e = mul_pair(z, make_float2(-1.44269504088896341f, -1.44269504088896341f)), r;
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
  e = add_pair(e, make_float2(1.f, 1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
  return r;
}

// VEC neighbouring channels as pairs: two fp32 operations in one instruction.
template <int VEC> struct Pairs {
  static constexpr int N = (VEC + 1) / 2;
  float2 p[N];
  __device__ __forceinline__ void set(const float (&x)[VEC]) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = make_float2(x[2 * i], 2 * i + 1 < VEC ? x[2 * i + 1 < VEC ? 2 * i + 1 : 0] : 0.f);
  }
  __device__ __forceinline__ void get(float (&x)[VEC]) const {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = i & 1 ? p[i / 2].y : p[i / 2].x;
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = make_float2(0.f, 0.f);
  }
  __device__ __forceinline__ void add_product(const Pairs& a, const Pairs& b) {        // += a b
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = fma_pair(a.p[i], b.p[i], p[i]);
  }
};
template <typename T, int VEC> __device__ __forceinline__ Pairs<VEC> widen(const Entries<T, VEC>& e) {
  float x[VEC];
  e.get(x);
  Pairs<VEC> r;
  r.set(x);
  return r;
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

// The taps and bias of VEC channels.  Where the weights of a thread are whole 16-byte units they are loaded as such (`wide`).
template <typename T, int W, int VEC>
__device__ __forceinline__ void load_taps(const ShortConv& a, int c, bool wide, Pairs<VEC> (&w)[W], Pairs<VEC>& bias) {
  constexpr int PER = 16 / sizeof(T), UNITS = W * VEC / PER;
  const T* wt = static_cast<const T*>(a.weight) + (size_t)c * W;
  float f[W * VEC], b[VEC];
  if (UNITS * PER == W * VEC && wide) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      Entries<T, PER> e;
      float x[PER];
      e.load(wt + u * PER);
      e.get(x);
#pragma unroll
      for (int i = 0; i < PER; ++i) f[u * PER + i] = x[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < W * VEC; ++i) f[i] = to_f32<T>(wt[i]);
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) b[i] = a.bias != nullptr ? to_f32<T>(static_cast<const T*>(a.bias)[c + i]) : 0.f;
#pragma unroll
  for (int j = 0; j < W; ++j) {
    float x[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = f[i * W + j];
    w[j].set(x);
  }
  bias.set(b);
}

template <typename T, int W, int VEC>
__global__ void __launch_bounds__(kThreads) short_conv_kernel(const __grid_constant__ ShortConv a, int groups, int col_blocks, int segs,
                                                              int seg_tokens, bool wide) {
  wait_for_kernels_ahead();
  const Place p = place(groups, VEC, col_blocks, segs, (long long)a.B * segs);
  if (!p.on) return;
  const int len = sequence_length(a.lengths, p.b, a.T);
  const T* x = reinterpret_cast<const T*>(a.x.p) + (long long)p.b * a.x.s0 + p.c;
  T* y = reinterpret_cast<T*>(a.out.p) + (long long)p.b * a.out.s0 + p.c;
  const int t0 = p.seg * seg_tokens, t1 = min(t0 + seg_tokens, a.T), live = min(t1, len);
  // whole steps of kAhead live tokens, then the rest one by one
  const int whole = live > t0 ? t0 + (live - t0) / kAhead * kAhead : t0;
  const T* px = x + (long long)t0 * a.x.s1;
  T* py = y + (long long)t0 * a.out.s1;
  Entries<T, VEC> in[kAhead];
  if (t0 < whole) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) in[u].load(px + u * a.x.s1);
  }
  Pairs<VEC> w[W], bias, win[W - 1];
  load_taps<T, W, VEC>(a, p.c, wide, w, bias);
  const size_t state = ((size_t)p.b * a.D + p.c) * (W - 1);
  if (p.seg == 0) {
    // the inputs before the first token, and those that the next call finds there (the same thread reads and writes a state)
    const T* s0 = static_cast<const T*>(a.s_init);
    float before[W - 1][VEC];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) before[j][i] = s0 != nullptr ? to_f32<T>(s0[state + i * (W - 1) + j]) : 0.f;
      win[j].set(before[j]);
    }
    if (a.s_final != nullptr) {
      T* s1 = static_cast<T*>(a.s_final);
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        const int t = len - (W - 1) + j;
        float v[VEC];
        if (t >= 0) {
          Entries<T, VEC> e;
          e.load(x + (long long)t * a.x.s1);
          e.get(v);
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int o = 0; o < W - 1; ++o)
              if (o == t + W - 1) v[i] = before[o][i];
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) s1[state + i * (W - 1) + j] = from_f32<T>(v[i]);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int t = t0 - (W - 1) + j;
      Entries<T, VEC> e;
      e.zero();
      if (t < len) e.load(x + (long long)t * a.x.s1);
      win[j] = widen<T, VEC>(e);
    }
  }
  auto emit = [&](const Pairs<VEC>& now, T* to) {
    Pairs<VEC> z = bias;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) z.add_product(w[j], win[j]);
    z.add_product(w[W - 1], now);
#pragma unroll
    for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
    win[W - 2] = now;
    float o[VEC];
    z.get(o);
    if (a.silu) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = silu_of<T>(o[i]);
    }
    Entries<T, VEC> e;
    e.set(o);
    e.store(to);
  };
  int t = t0;
#pragma unroll 2
  for (; t < whole; t += kAhead) {
    Entries<T, VEC> next[kAhead];
    px += kAhead * a.x.s1;
    if (t + kAhead < whole) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) next[u].load(px + u * a.x.s1);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) emit(widen<T, VEC>(in[u]), py + u * a.out.s1);
    py += kAhead * a.out.s1;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) in[u] = next[u];
  }
#pragma unroll 1
  for (; t < t1; ++t, px += a.x.s1, py += a.out.s1) {
    Entries<T, VEC> e;
    e.zero();
    if (t < live) {
      e.load(px);
      emit(widen<T, VEC>(e), py);
    } else {
      e.store(py);
    }
  }
}

// part: [blocks of segments][W + 1][D], or null where no sum is wanted
template <typename T, int W, int VEC>
__global__ void __launch_bounds__(kThreads) short_conv_bwd_kernel(const __grid_constant__ ShortConv a, int groups, int col_blocks, int segs,
                                                                  int seg_tokens, bool wide, float* __restrict__ part) {
  extern __shared__ float red[];       // [ty][W + 1][tx * VEC]
  wait_for_kernels_ahead();
  const Place p = place(groups, VEC, col_blocks, segs, (long long)a.B * segs);
  Pairs<VEC> dw[W], db;
#pragma unroll
  for (int j = 0; j < W; ++j) dw[j].zero();
  db.zero();
  if (p.on) {
    const int len = sequence_length(a.lengths, p.b, a.T);
    const T* x = reinterpret_cast<const T*>(a.x.p) + (long long)p.b * a.x.s0 + p.c;
    const T* dy = reinterpret_cast<const T*>(a.dout.p) + (long long)p.b * a.dout.s0 + p.c;
    T* dx = reinterpret_cast<T*>(a.dx.p) + (long long)p.b * a.dx.s0 + p.c;
    const int t0 = p.seg * seg_tokens, t1 = min(t0 + seg_tokens, a.T), live = min(t1, len);
    const int whole = live > t0 ? t0 + (live - t0) / kAhead * kAhead : t0;
    const T *px = x + (long long)t0 * a.x.s1, *pg = dy + (long long)t0 * a.dout.s1;
    T* po = dx + (long long)(t0 - (W - 1)) * a.dx.s1;            // of the input that the token in hand is the last tap of
    Entries<T, VEC> in[kAhead], gin[kAhead];
    if (t0 < whole) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        in[u].load(px + u * a.x.s1);
        gin[u].load(pg + u * a.dout.s1);
      }
    }
    Pairs<VEC> w[W], bias, win[W - 1], gw[W - 1];
    load_taps<T, W, VEC>(a, p.c, wide, w, bias);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int t = t0 - (W - 1) + j;
      Entries<T, VEC> e;
      e.zero();
      if (t >= 0 && t < len) e.load(x + (long long)t * a.x.s1);
      win[j] = widen<T, VEC>(e);
      gw[j].zero();
    }
    // One token: the gradient before the activation; into the sums where the token is this segment's; the input W - 1 tokens back, which
    // has met all its taps, where it is.
    auto emit = [&](const Pairs<VEC>& now, Pairs<VEC> g, bool own, bool store, bool zero, T* to) {
      if (a.silu) {
        Pairs<VEC> z = bias;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) z.add_product(w[j], win[j]);
        z.add_product(w[W - 1], now);
        float zz[VEC], gg[VEC];
        z.get(zz);
        g.get(gg);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float sig = sigmoid_of<T>(zz[i]);
          gg[i] *= fmaf(zz[i] * sig, 1.f - sig, sig);            // sigmoid (1 + z (1 - sigmoid)); z sigmoid is finite where z is
        }
        g.set(gg);
      }
      if (own) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) dw[j].add_product(g, win[j]);
        dw[W - 1].add_product(g, now);
#pragma unroll
        for (int i = 0; i < Pairs<VEC>::N; ++i) db.p[i] = add_pair(db.p[i], g.p[i]);
      }
      if (store) {
        Pairs<VEC> out;
#pragma unroll
        for (int i = 0; i < Pairs<VEC>::N; ++i) out.p[i] = mul_pair(w[0].p[i], g.p[i]);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) out.add_product(w[W - 1 - j], gw[j]);
        float o[VEC];
        out.get(o);
        Entries<T, VEC> e;
        e.set(o);
        if (zero) e.zero();
        e.store(to);
      }
#pragma unroll
      for (int j = 0; j + 1 < W - 1; ++j) {
        win[j] = win[j + 1];
        gw[j] = gw[j + 1];
      }
      win[W - 2] = now;
      gw[W - 2] = g;
    };
    int t = t0;
#pragma unroll 1
    for (; t < whole; t += kAhead) {
      Entries<T, VEC> next[kAhead], gnext[kAhead];
      px += kAhead * a.x.s1;
      pg += kAhead * a.dout.s1;
      if (t + kAhead < whole) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          next[u].load(px + u * a.x.s1);
          gnext[u].load(pg + u * a.dout.s1);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) emit(widen<T, VEC>(in[u]), widen<T, VEC>(gin[u]), true, t + u >= t0 + W - 1, false, po + u * a.dx.s1);
      po += kAhead * a.dx.s1;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        in[u] = next[u];
        gin[u] = gnext[u];
      }
    }
#pragma unroll 1
    for (; t < t1 + W - 1; ++t, px += a.x.s1, pg += a.dout.s1, po += a.dx.s1) {
      Entries<T, VEC> e, g;
      e.zero();
      g.zero();                                                  // (nothing behind the sequence's end has a gradient)
      if (t < min(t1 + W - 1, len)) {
        e.load(px);
        g.load(pg);
      }
      const int at = t - (W - 1);
      emit(widen<T, VEC>(e), widen<T, VEC>(g), t < live, at >= t0 && at < t1, at >= len, po);
    }
  }
  if (part == nullptr) return;
  const int cols = blockDim.x * VEC;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    float v[VEC];
    if (j < W) dw[j < W ? j : 0].get(v);
    else db.get(v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) red[((size_t)threadIdx.y * (W + 1) + j) * cols + threadIdx.x * VEC + i] = v[i];
  }
  __syncthreads();
  const unsigned cb = blockIdx.x % (unsigned)col_blocks, rb = blockIdx.x / (unsigned)col_blocks;
  for (int e = threadIdx.y * blockDim.x + threadIdx.x; e < (W + 1) * cols; e += blockDim.x * blockDim.y) {
    float sum = 0.f;
    for (int y = 0; y < (int)blockDim.y; ++y) sum += red[(size_t)y * (W + 1) * cols + e];
    const int j = e / cols, c = (int)cb * cols + e % cols;
    if (c < a.D) part[((size_t)rb * (W + 1) + j) * a.D + c] = sum;
  }
}

// ---- rows of whole 16-byte units, sequences of some length: tiles through shared memory ----
// The walk above has a few loads of 4 bytes per thread in flight, and its time is their latency (8 x 4096 x 1024 bf16: forward 47 us,
// with the gradients 132).  Here a block asks for its whole tile at once by asynchronous copies of 16 bytes, which also put zeros where a
// token is not the sequence's, and several blocks share an SM; a thread then walks a run of tokens of two channels in shared memory.
constexpr int kRun = 32, kBwdRun = 16;         // (the backward has twice two tensors of a tile in shared memory)

__device__ __forceinline__ void copy_row_unit(void* smem, const void* src, bool on) {
  const uint32_t n = on ? 16u : 0u;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// Asks for `rows` rows of 2 tx channels from token t on (t may be negative); tokens outside 0 .. live - 1 and channels from D on
// become zeros.  shift: log2 of the 16-byte units of a row.
template <typename T>
__device__ __forceinline__ void ask_rows(unsigned char* smem, const View& v, int b, int t, int rows, int live, int c0, int D, int shift) {
  constexpr int E = 16 / sizeof(T);
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, down = (int)(blockDim.x * blockDim.y) >> shift;
  const int c = c0 + (tid & ((1 << shift) - 1)) * E;
  const T* base = reinterpret_cast<const T*>(v.p) + (long long)b * v.s0;
  int r = tid >> shift;
  const T* from = base + (long long)(t + r) * v.s1 + c;
  const long long step = (long long)down * v.s1;
  unsigned char* to = smem + (size_t)tid * 16;
  for (; r < rows; r += down, from += step, to += (size_t)down << (shift + 4)) {
    const bool on = (unsigned)(t + r) < (unsigned)live && c < D;
    copy_row_unit(to, on ? from : base, on);
  }
}

struct Tile {
  int b, t0, c0, c;
  unsigned cb;
};
__device__ __forceinline__ Tile tile_at(unsigned index, int tiles, int tile_tokens, unsigned cb) {
  Tile t;
  t.b = (int)(index / (unsigned)tiles);
  t.t0 = (int)(index - (unsigned)t.b * (unsigned)tiles) * tile_tokens;
  t.cb = cb;
  t.c0 = (int)cb * blockDim.x * 2;
  t.c = t.c0 + threadIdx.x * 2;
  return t;
}

template <typename T, int W, bool SILU>
__global__ void __launch_bounds__(kThreads) short_conv_tile_kernel(const __grid_constant__ ShortConv a, int col_blocks, int tiles, int shift, bool wide) {
  extern __shared__ __align__(16) unsigned char smem[];          // [tile + W - 1 tokens][2 tx channels]
  wait_for_kernels_ahead();
  const int tile_tokens = blockDim.y * kRun;
  const Tile p = tile_at(blockIdx.x / (unsigned)col_blocks, tiles, tile_tokens, blockIdx.x % (unsigned)col_blocks);
  const int len = sequence_length(a.lengths, p.b, a.T);
  ask_rows<T>(smem, a.x, p.b, p.t0 - (W - 1), tile_tokens + W - 1, len, p.c0, a.D, shift);
  commit_copies();
  const bool on = p.c < a.D;
  Pairs<2> w[W], bias;
  if (on) load_taps<T, W, 2>(a, p.c, wide, w, bias);
  wait_copies<0>();
  __syncthreads();
  T* rows = reinterpret_cast<T*>(smem);
  const int width = blockDim.x * 2;
  if (p.t0 == 0 && (a.s_init != nullptr || a.s_final != nullptr)) {
    // the inputs before the first token, and those that the next call finds there (the same thread reads and writes a state)
    if (threadIdx.y == 0 && on) {
      const T *s0 = static_cast<const T*>(a.s_init), *x = reinterpret_cast<const T*>(a.x.p) + (long long)p.b * a.x.s0;
      T* s1 = static_cast<T*>(a.s_final);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const size_t state = ((size_t)p.b * a.D + p.c + i) * (W - 1);
        T before[W - 1], after[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
          before[j] = s0 != nullptr ? s0[state + j] : from_f32<T>(0.f);
          rows[j * width + threadIdx.x * 2 + i] = before[j];
        }
        if (s1 != nullptr) {
#pragma unroll
          for (int j = 0; j < W - 1; ++j) {
            const int t = len - (W - 1) + j;
            after[j] = from_f32<T>(0.f);
            if (t >= 0) after[j] = x[(long long)t * a.x.s1 + p.c + i];
#pragma unroll
            for (int o = 0; o < W - 1; ++o)
              if (o == t + W - 1) after[j] = before[o];
          }
#pragma unroll
          for (int j = 0; j < W - 1; ++j) s1[state + j] = after[j];
        }
      }
    }
    __syncthreads();
  }
  if (!on) return;
  const T* r = rows + (size_t)threadIdx.y * kRun * width + threadIdx.x * 2;
  auto at = [&](int row) {
    Entries<T, 2> e;
    e.load(r + (size_t)row * width);
    return widen<T, 2>(e);
  };
  Pairs<2> win[W - 1];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) win[j] = at(j);
  const int t0 = p.t0 + threadIdx.y * kRun;
  T* y = reinterpret_cast<T*>(a.out.p) + (long long)p.b * a.out.s0 + (long long)t0 * a.out.s1 + p.c;
  auto token = [&](int u, bool checked) {
    const Pairs<2> now = at(W - 1 + u);
    Pairs<2> z = bias;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) z.add_product(w[j], win[j]);
    z.add_product(w[W - 1], now);
#pragma unroll
    for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
    win[W - 2] = now;
    float2 v = z.p[0];
    if (SILU) v = sizeof(T) == 4 ? make_float2(silu_of<T>(v.x), silu_of<T>(v.y)) : mul_pair(v, sigmoid_pair<T>(v));
    const float o[2] = {v.x, v.y};
    Entries<T, 2> e;
    e.set(o);
    if (checked && t0 + u >= len) e.zero();
    if (!checked || t0 + u < a.T) e.store(y);
    y += a.out.s1;
  };
  if (t0 + kRun <= len) {
#pragma unroll 8
    for (int u = 0; u < kRun; ++u) token(u, false);
  } else {
#pragma unroll 1
    for (int u = 0; u < kRun; ++u) token(u, true);
  }
}

// A block has one group of channels and every gridDim.y-th tile: the next tile is on its way while one is worked on, and the sums of
// the weights stay in registers.  8 x 4096 x 1024: 70.8 us (floor 30.8), with the forward 95.9 (51), bound by instructions and their latency
// (122 registers).  Two of them are what keeps the rows behind the end zero and out of the sums; a loop of its own for the runs at the
// end took 72.4 and, with lengths between 1 and 4096, 83 instead of 50 to 59.  Not kept, measured before that with the forward (94 then): three
// and four blocks on an SM (97, 93), a run's last gradients from the next run through shared memory instead of once more (96), the
// sigmoid's constants in scalar instructions (95).  part: [gridDim.y][W + 1][D], or null
template <typename T, int W, bool SILU>
__global__ void __launch_bounds__(kThreads, 2) short_conv_bwd_tile_kernel(const __grid_constant__ ShortConv a, int tiles, unsigned n_tiles, int shift, bool wide,
                                                                          float* __restrict__ part) {
  extern __shared__ __align__(16) unsigned char smem[];          // 2 x {x: [tile + 2 (W - 1)], dy: [tile + W - 1]}[2 tx channels]
  wait_for_kernels_ahead();
  const int tile_tokens = blockDim.y * kBwdRun, width = blockDim.x * 2;
  const int x_rows = tile_tokens + 2 * (W - 1), g_rows = tile_tokens + W - 1;
  const size_t g_at = (size_t)x_rows << (shift + 4), buffer = (size_t)(x_rows + g_rows) << (shift + 4);
  auto ask = [&](unsigned index, unsigned char* to) {
    const Tile p = tile_at(index, tiles, tile_tokens, blockIdx.x);
    const int len = sequence_length(a.lengths, p.b, a.T);
    ask_rows<T>(to, a.x, p.b, p.t0 - (W - 1), x_rows, len, p.c0, a.D, shift);
    ask_rows<T>(to + g_at, a.dout, p.b, p.t0, g_rows, len, p.c0, a.D, shift);
  };
  Pairs<2> dw[W], db, w[W], bias;
#pragma unroll
  for (int j = 0; j < W; ++j) dw[j].zero();
  db.zero();
  const int c = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 2;
  const bool on = c < a.D;
  unsigned index = blockIdx.y;
  if (index < n_tiles) ask(index, smem);
  commit_copies();
  if (on) load_taps<T, W, 2>(a, c, wide, w, bias);
  for (int k = 0; index < n_tiles; index += gridDim.y, k ^= 1) {
    if (index + gridDim.y < n_tiles) ask(index + gridDim.y, smem + (k ^ 1) * buffer);
    commit_copies();
    wait_copies<1>();
    __syncthreads();
    const Tile p = tile_at(index, tiles, tile_tokens, blockIdx.x);
    const int t0 = p.t0 + threadIdx.y * kBwdRun, len = sequence_length(a.lengths, p.b, a.T);
    if (on && t0 < len) {
      const T* xr = reinterpret_cast<const T*>(smem + k * buffer) + (size_t)threadIdx.y * kBwdRun * width + threadIdx.x * 2;
      const T* gr = reinterpret_cast<const T*>(smem + k * buffer + g_at) + (size_t)threadIdx.y * kBwdRun * width + threadIdx.x * 2;
      auto get = [&](const T* rows, int row) {
        Entries<T, 2> e;
        e.load(rows + (size_t)row * width);
        return widen<T, 2>(e);
      };
      const int left = len - t0;                                 // tokens of the sequence: no others count in the sums (0 times inf is NaN)
      Pairs<2> win[W - 1], gw[W - 1];
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        win[j] = get(xr, j);
        gw[j].zero();
      }
      T* to = reinterpret_cast<T*>(a.dx.p) + (long long)p.b * a.dx.s0 + (long long)(t0 - (W - 1)) * a.dx.s1 + c;
      // One token: the gradient before the activation (zero where the token is not the sequence's: dy is); own: into the sums; store:
      // the input W - 1 tokens back has met all its taps.
      auto token = [&](int u, bool own, bool store) {
        const Pairs<2> now = get(xr, W - 1 + u);
        Pairs<2> g = get(gr, u);
        if (SILU) {
          Pairs<2> z = bias;
#pragma unroll
          for (int j = 0; j < W - 1; ++j) z.add_product(w[j], win[j]);
          z.add_product(w[W - 1], now);
          // sigmoid (1 + z (1 - sigmoid)); z sigmoid is finite where z is
          const float2 sig = sigmoid_pair<T>(z.p[0]), rest = fma_pair(sig, make_float2(-1.f, -1.f), make_float2(1.f, 1.f));
          g.p[0] = mul_pair(g.p[0], fma_pair(mul_pair(z.p[0], sig), rest, sig));
        }
        if (own && u < left) {
#pragma unroll
          for (int j = 0; j < W - 1; ++j) dw[j].add_product(g, win[j]);
          dw[W - 1].add_product(g, now);
          db.p[0] = add_pair(db.p[0], g.p[0]);
        }
        if (store) {
          Pairs<2> out;
          out.p[0] = mul_pair(w[0].p[0], g.p[0]);
#pragma unroll
          for (int j = 0; j < W - 1; ++j) out.add_product(w[W - 1 - j], gw[j]);
          const float o[2] = {out.p[0].x, out.p[0].y};
          Entries<T, 2> e;
          e.set(o);
          if (t0 + u - (W - 1) < a.T) e.store(to);
        }
        to += a.dx.s1;
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) {
          win[j] = win[j + 1];
          gw[j] = gw[j + 1];
        }
        win[W - 2] = now;
        gw[W - 2] = g;
      };
#pragma unroll
      for (int u = 0; u < W - 1; ++u) token(u, true, false);
#pragma unroll
      for (int u = W - 1; u < kBwdRun; ++u) token(u, true, true);
#pragma unroll
      for (int u = kBwdRun; u < kBwdRun + W - 1; ++u) token(u, false, true);
    }
    // Rows behind the end.  (The last run has stored some: zeros, but NaN where an input before the end is not finite.)
    if (on && a.lengths != nullptr) {
      T* to = reinterpret_cast<T*>(a.dx.p) + (long long)p.b * a.dx.s0 + c;
      Entries<T, 2> e;
      e.zero();
#pragma unroll 1
      for (int t = max(t0, len); t < min(t0 + kBwdRun, a.T); ++t) e.store(to + (long long)t * a.dx.s1);
    }
    __syncthreads();                                             // the buffer may be asked into again
  }
  if (part == nullptr) return;
  wait_copies<0>();
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);                   // [ty][W + 1][2 tx]
#pragma unroll
  for (int j = 0; j <= W; ++j)
    *reinterpret_cast<float2*>(red + ((size_t)threadIdx.y * (W + 1) + j) * width + threadIdx.x * 2) = j < W ? dw[j < W ? j : 0].p[0] : db.p[0];
  __syncthreads();
  for (int e = threadIdx.y * blockDim.x + threadIdx.x; e < (W + 1) * width; e += blockDim.x * blockDim.y) {
    float sum = 0.f;
    for (int y = 0; y < (int)blockDim.y; ++y) sum += red[(size_t)y * (W + 1) * width + e];
    const int j = e / width, col = (int)blockIdx.x * width + e % width;
    if (col < a.D) part[((size_t)blockIdx.y * (W + 1) + j) * a.D + col] = sum;
  }
}

// dweight[c][j] and dbias[c]: the blocks' sums added in order, eight runs of them side by side, eight loads of a run in flight (forward
// and backward of 16 x 31 x 1024: 11.3 us, one load at a time 13.0).
__global__ void __launch_bounds__(256) short_conv_sum_kernel(const float* __restrict__ part, int blocks, int W, int D,
                                                             float* __restrict__ dweight, float* __restrict__ dbias) {
  __shared__ float red[8][33];
  wait_for_kernels_ahead();
  const int e = blockIdx.x * 32 + threadIdx.x, n = (W + 1) * D;
  float sum = 0.f;
  if (e < n)
#pragma unroll 8
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
// Segments of 32 tokens; shorter ones (down to 8, backward 16: its sums are per segment) while there are fewer threads than the GPU
// holds.  Measured, us, bf16, segments of 8 / 16 / 32 / 64: 1 x 4096 x 1000 channels forward 6.1 / 6.7 / 8.0 / 8.8, backward 18.3 / 13.5 /
// 17.6 / 27.5; 8 x 4096 x 1000 forward 44.5 / 41.0 / 39.2 / 46.2, backward 147 / 106 / 85 / 85.
ConvGrid conv_grid(int B, int T, int D, int vec, bool backward) {
  ConvGrid g;
  g.groups = (D + vec - 1) / vec;
  int tx = 1;
  while (tx < g.groups && tx < 64) tx *= 2;
  g.block = dim3(tx, kThreads / tx);
  g.col_blocks = (g.groups + tx - 1) / tx;
  g.seg_tokens = 32;
  while (g.seg_tokens > (backward ? 16 : 8) && (double)g.groups * B * ((T + g.seg_tokens - 1) / g.seg_tokens) < kPlanSMs * 1024.0) g.seg_tokens /= 2;
  g.segs = (T + g.seg_tokens - 1) / g.seg_tokens;
  g.row_blocks = ((long long)B * g.segs + g.block.y - 1) / g.block.y;
  return g;
}

bool conv_aligned(const ShortConv& a, const View& v, int bytes) {
  const long long e = a.dtype == KATA_F32 ? 4 : 2;
  return (reinterpret_cast<uintptr_t>(v.p) % bytes) == 0 && (v.s0 * e) % bytes == 0 && (v.s1 * e) % bytes == 0;
}

bool taps_aligned(const ShortConv& a) { return (reinterpret_cast<uintptr_t>(a.weight) & 15u) == 0; }

// Tiles: 64 channel pairs (32 of fp32) x 4 runs of tokens, or more runs of fewer pairs.
struct TileGrid {
  int tx, ty, col_blocks, tiles, shift;
  long long n_tiles;
  int walkers;                         // blocks that share out the tiles of a group of channels in the backward
};
TileGrid tile_grid(int B, int T, int D, int elem, int run) {
  TileGrid g;
  const int most = elem == 2 ? 64 : 32;
  g.tx = 1;
  while (g.tx < most && g.tx * 2 < D) g.tx *= 2;
  g.ty = most * 4 / g.tx;
  g.col_blocks = (D + 2 * g.tx - 1) / (2 * g.tx);
  g.tiles = (T + g.ty * run - 1) / (g.ty * run);
  g.n_tiles = (long long)B * g.tiles;
  g.shift = 0;
  while ((16 << g.shift) < 2 * g.tx * elem) ++g.shift;
  const long long share = (3 * kPlanSMs + g.col_blocks - 1) / g.col_blocks;
  g.walkers = (int)(share < g.n_tiles ? share : g.n_tiles);
  if (g.walkers > 65535) g.walkers = 65535;
  return g;
}
// Tiles need rows of whole 16-byte units, a size that is worth their start, and sequences that fill them: a tile has 128 tokens (backward
// 64) of 128 channels or more, twice as many of half as many, and so on.
// Measured, us, walk / tiles, 1024 channels, 32768 tokens unless others are named:
//   forward, bf16: T = 64: 47 / 49, 128: 48 / 27, 16384: 47 / 27; 4096 tokens: 6.8 / 6.3, 1024 tokens: 3.8 / 4.4
//   forward, fp32: T = 64: 66 / 90, 128: 66 / 48; 8192 tokens: 17.5 / 16.4, 4096 tokens: 9.4 / 10.8
//   backward, bf16, sequences x T: 512 x 32: 46 / 46, 128 x 32: 14 / 17, 512 x 48: 77 / 70, 256 x 64: 47 / 38, 8 x 4096: 82 / 71; in rounds of
//   tiles: 64 x 128 (more than two) 26 / 22, 32 x 128 (the second nearly empty) 14.3 / 14.4, 16 x 128 (one) 11.9 / 9.0
//   backward, fp32 (with the forward, less the forward): 16384 tokens 69 / 82, 32768: 120 / 161: never tiles
// Fewer channels, 2^24 entries, and how full the tiles are (channels x T):
//   forward, bf16: full 16 x 1024 16.6 / 13.4, 64 x 256 19.4 / 13.4, three quarters 16 x 768 16.7 / 19.0, 64 x 192 17.4 / 19.0, 1024 x 192 18.2 /
//   19.0, half 64 x 128 19.3 / 26.0, an eighth 16 x 128 17.5 / 100; eight channels 8 x 2048 (full) 22.1 / 20.9, 8 x 128 22.6 / 220
//   forward, fp32: full 16 x 512 37.6 / 28.8, three quarters 16 x 384 37.8 / 35.0, 64 x 192 34.1 / 34.5, half 16 x 256 38.0 / 47.6, 64 x 64 34.4 / 47.6
//   backward, bf16: full 16 x 512 44 / 35, half 16 x 256 44 / 42, 32 x 128 50 / 42, 64 x 64 49 / 42, 3/8 16 x 192 44 / 51, an eighth 16 x 64 44 / 119;
//   eight channels, full 8 x 1024 44 / 48, 8 x 64 44 / 229
bool use_tiles(const ShortConv& a, bool backward) {
  const int e = a.dtype == KATA_F32 ? 4 : 2;
  if ((a.D * e) % 16 != 0 || a.D < 16 || !conv_aligned(a, a.x, 16)) return false;
  if (backward && (e != 2 || !conv_aligned(a, a.dout, 16))) return false;
  const int run = backward ? kBwdRun : kRun;
  const TileGrid g = tile_grid(a.B, a.T, a.D, e, run);
  const double full = (double)a.T / ((double)g.tiles * g.ty * run);
  if (!backward) return a.T >= 128 && full >= (e == 2 ? 0.8 : 0.7) && (double)a.B * a.T * a.D >= (e == 2 ? 1 << 21 : 1 << 23);
  return a.T >= 48 && full >= 0.5 && (g.n_tiles <= g.walkers || g.n_tiles >= 2 * g.walkers);
}

template <typename T, int W, bool SILU> void launch_tiles(const ShortConv& a, LaunchCtx& ctx) {
  const TileGrid g = tile_grid(a.B, a.T, a.D, sizeof(T), kRun);
  const size_t smem = (size_t)(g.ty * kRun + W - 1) << (g.shift + 4);
  launch_after(ctx, short_conv_tile_kernel<T, W, SILU>, dim3((unsigned)(g.n_tiles * g.col_blocks)), dim3(g.tx, g.ty), smem, a, g.col_blocks, g.tiles, g.shift,
               taps_aligned(a));
}

template <typename T, int W, bool SILU> void launch_bwd_tiles(const ShortConv& a, float* ws, LaunchCtx& ctx) {
  const TileGrid g = tile_grid(a.B, a.T, a.D, sizeof(T), kBwdRun);
  const bool sums = a.dweight != nullptr || a.dbias != nullptr;
  const size_t tile = (size_t)(2 * (g.ty * kBwdRun) + 3 * (W - 1)) << (g.shift + 4);
  const size_t red = (size_t)g.ty * (W + 1) * 2 * g.tx * sizeof(float);
  const size_t smem = 2 * tile > red ? 2 * tile : red;
  if (!allow_smem<short_conv_bwd_tile_kernel<T, W, SILU>>(160 * 1024)) {
    ctx.status = KATA_ERR_CUDA;
    return;
  }
  launch_after(ctx, short_conv_bwd_tile_kernel<T, W, SILU>, dim3(g.col_blocks, g.walkers), dim3(g.tx, g.ty), smem, a, g.tiles, (unsigned)g.n_tiles, g.shift, taps_aligned(a),
               sums ? ws : nullptr);
  if (sums)
    launch_after(ctx, short_conv_sum_kernel, dim3(((W + 1) * a.D + 31) / 32), dim3(32, 8), 0, ws, g.walkers, W, a.D, a.dweight, a.dbias);
}

template <typename T, int W, int VEC> void launch_fwd(const ShortConv& a, LaunchCtx& ctx) {
  const ConvGrid g = conv_grid(a.B, a.T, a.D, VEC, false);
  launch_after(ctx, short_conv_kernel<T, W, VEC>, dim3((unsigned)(g.row_blocks * g.col_blocks)), g.block, 0, a, g.groups, g.col_blocks, g.segs, g.seg_tokens, taps_aligned(a));
}

template <typename T, int W, int VEC> void launch_bwd(const ShortConv& a, float* ws, LaunchCtx& ctx) {
  const ConvGrid g = conv_grid(a.B, a.T, a.D, VEC, true);
  const bool sums = a.dweight != nullptr || a.dbias != nullptr;
  const size_t smem = sums ? (size_t)kThreads * VEC * (W + 1) * sizeof(float) : 0;
  launch_after(ctx, short_conv_bwd_kernel<T, W, VEC>, dim3((unsigned)(g.row_blocks * g.col_blocks)), g.block, smem, a, g.groups, g.col_blocks, g.segs,
               g.seg_tokens, taps_aligned(a), sums ? ws : nullptr);
  if (sums)
    launch_after(ctx, short_conv_sum_kernel, dim3(((W + 1) * a.D + 31) / 32), dim3(32, 8), 0, ws, (int)g.row_blocks, W, a.D, a.dweight, a.dbias);
}

constexpr int kVec = 2;                // channels per thread

template <typename T, int W> void dispatch(const ShortConv& a, bool backward, float* ws, LaunchCtx& ctx) {
  constexpr int bytes = kVec * sizeof(T);
  if (backward) {
    const bool pairs = a.D % kVec == 0 && conv_aligned(a, a.dx, bytes);
    if constexpr (sizeof(T) == 2) {
      if (pairs && use_tiles(a, true)) return a.silu ? launch_bwd_tiles<T, W, true>(a, ws, ctx) : launch_bwd_tiles<T, W, false>(a, ws, ctx);
    }
    if (pairs && conv_aligned(a, a.x, bytes) && conv_aligned(a, a.dout, bytes)) launch_bwd<T, W, kVec>(a, ws, ctx);
    else launch_bwd<T, W, 1>(a, ws, ctx);
  } else {
    const bool pairs = a.D % kVec == 0 && conv_aligned(a, a.out, bytes);
    if (pairs && use_tiles(a, false)) a.silu ? launch_tiles<T, W, true>(a, ctx) : launch_tiles<T, W, false>(a, ctx);
    else if (pairs && conv_aligned(a, a.x, bytes)) launch_fwd<T, W, kVec>(a, ctx);
    else launch_fwd<T, W, 1>(a, ctx);
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

// (the most of all ways to read rows: the scratch depends on sizes alone)
size_t short_conv_bwd_workspace_elems(int B, int T, int D, int W) {
  long long most = conv_grid(B, T, D, 1, true).row_blocks;
  const long long others[2] = {conv_grid(B, T, D, kVec, true).row_blocks, tile_grid(B, T, D, 2, kBwdRun).walkers};
  for (const long long o : others)
    if (o > most) most = o;
  return (size_t)most * (W + 1) * D;
}

void short_conv_bwd(const ShortConv& a, float* ws, LaunchCtx& ctx) { run(a, true, ws, ctx); }

}  // namespace kata
