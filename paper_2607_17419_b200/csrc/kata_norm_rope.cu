// Norm of query and key rows by their root mean square and rotation by their positions, and the backward of both:
//   y = R_p (w * x r),  r = 1 / sqrt(mean(x^2) + eps)
//   u = R_p^T dy,  dw = sum u * x r,  dx = r (u * w - x r mean(u * w * x r))
// HBM-bound: every row is read and written once (backward: two reads, one write).  A row is held by d / (16 bytes) neighbouring
// lanes.  A lane has both sides of its pairs, as two pieces of 8 bytes, so nothing but the sums of a row crosses lanes.  The turn of
// a pair depends on the token and not on the head: the lanes of a token form their sines once and walk the heads with them.
// Arithmetic goes two entries at a time.  8 x 4096 tokens, 32 heads of 64: forward 48.5 us in bf16 and 87 in fp32, 0.85 and 0.94 of the
// copy bandwidth; backward 108 and 164 (floor 61.5 and 123), pairs of neighbours 88 and 147.  The backward is bound by the latency of
// its loads, with three blocks on an SM: the 80 registers that leaves spill 48 bytes in bf16 (neighbours 20), since a thread carries
// the sums and the walk of queries and of keys.  (Forward and backward in bf16, 671 MB, 161 us together; two blocks of the backward and
// three of the forward: 181; one head in flight less each: 164.)
// Angles: position times a 64-bit fraction of a turn, in wrapping integers: no rounding grows with the position.
#include "kata_rows.cuh"

namespace kata {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4, kBwdAhead = 2;                   // heads in flight
constexpr int kBlocks = 3 * kPlanSMs;                      // of the backward: what fits at once

// What a lane has of a row: entries e0 .. and e1 .. (N pairs of entries each).  Of half-split pairs e1 holds the other sides; of
// neighbouring ones the even entries of both pieces are one side.  Entries that are not turned fill the lanes behind.
template <typename T> struct Half {
  static constexpr int E = 8 / sizeof(T), N = E / 2;       // entries of a piece, pairs of them
};
struct Lane {
  int e0, e1;
  bool turned;
};
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ Lane lane_of(const NormRope& a, int lanes) {
  constexpr int E = Half<T>::E;
  const int l = threadIdx.x & (lanes - 1), turning = a.rot / (2 * E);
  Lane r;
  r.turned = l < turning;
  r.e0 = NEIGHBOURS || !r.turned ? 2 * E * l : E * l;
  r.e1 = NEIGHBOURS || !r.turned ? r.e0 + E : a.rot / 2 + E * l;
  return r;
}

// The two sides of a lane's pairs, as fp32 in twos.
template <typename T> struct Sides {
  static constexpr int N = Half<T>::N;
  float2 a[N], b[N];
};
template <typename T> struct Pieces {
  Entries<T, Half<T>::E> p, q;
  __device__ __forceinline__ void load(const T* row, const Lane& ln) {
    p.load(row + ln.e0);
    q.load(row + ln.e1);
  }
  __device__ __forceinline__ void store(T* row, const Lane& ln) const {
    p.store(row + ln.e0);
    q.store(row + ln.e1);
  }
  __device__ __forceinline__ void zero() {
    p.zero();
    q.zero();
  }
  template <bool NEIGHBOURS> __device__ __forceinline__ Sides<T> get() const {
    constexpr int E = Half<T>::E, N = Half<T>::N;
    float x[E], y[E];
    p.get(x);
    q.get(y);
    Sides<T> s;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (NEIGHBOURS) {                                    // pairs (x0 x1) (x2 x3) .. (y0 y1) ..
        const int j = 4 * i;
        s.a[i] = make_float2(j < E ? x[j < E ? j : 0] : y[j < E ? 0 : j - E], j + 2 < E ? x[j + 2 < E ? j + 2 : 0] : y[j + 2 < E ? 0 : j + 2 - E]);
        s.b[i] = make_float2(j < E ? x[j < E ? j + 1 : 0] : y[j < E ? 0 : j + 1 - E], j + 2 < E ? x[j + 2 < E ? j + 3 : 0] : y[j + 2 < E ? 0 : j + 3 - E]);
      } else {
        s.a[i] = make_float2(x[2 * i], x[2 * i + 1]);
        s.b[i] = make_float2(y[2 * i], y[2 * i + 1]);
      }
    }
    return s;
  }
  template <bool NEIGHBOURS> __device__ __forceinline__ void set(const Sides<T>& s) {
    constexpr int E = Half<T>::E, N = Half<T>::N;
    float x[E], y[E];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (NEIGHBOURS) {
        const int j = 4 * i;
        const float v[4] = {s.a[i].x, s.b[i].x, s.a[i].y, s.b[i].y};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < E) x[j + k < E ? j + k : 0] = v[k];
          else y[j + k < E ? 0 : j + k - E] = v[k];
      } else {
        x[2 * i] = s.a[i].x;
        x[2 * i + 1] = s.a[i].y;
        y[2 * i] = s.b[i].x;
        y[2 * i + 1] = s.b[i].y;
      }
    }
    p.set(x);
    q.set(y);
  }
};

// cos and sin of this lane's pairs at a position.
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void turns_of(const unsigned long long* turns, const Lane& ln, long long pos, float2 (&c)[Half<T>::N], float2 (&s)[Half<T>::N]) {
  const int f = NEIGHBOURS ? ln.e0 / 2 : ln.e0;            // first pair
#pragma unroll
  for (int i = 0; i < Half<T>::N; ++i) {
    c[i] = make_float2(1.f, 1.f);
    s[i] = make_float2(0.f, 0.f);
    if (ln.turned) {
      // half turns in [-1, 1)
      sincospif((float)(int)(((unsigned long long)pos * turns[f + 2 * i]) >> 32) * 4.656612873077392578125e-10f, &s[i].x, &c[i].x);
      sincospif((float)(int)(((unsigned long long)pos * turns[f + 2 * i + 1]) >> 32) * 4.656612873077392578125e-10f, &s[i].y, &c[i].y);
    }
  }
}

template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ Sides<T> weights_of(const void* w, const Lane& ln) {
  constexpr int E = Half<T>::E;
  Sides<T> r;
  Pieces<T> x;
  float one[E];
#pragma unroll
  for (int i = 0; i < E; ++i) one[i] = 1.f;
  x.p.set(one);
  x.q.set(one);
  if (w != nullptr) {                                      // (entry by entry: weights have no alignment to keep)
    float u[E], v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      u[i] = to_f32<T>(static_cast<const T*>(w)[ln.e0 + i]);
      v[i] = to_f32<T>(static_cast<const T*>(w)[ln.e1 + i]);
    }
    x.p.set(u);
    x.q.set(v);
  }
  return x.template get<NEIGHBOURS>();
}

__device__ __forceinline__ float2 twice(float x) { return make_float2(x, x); }
__device__ __forceinline__ float row_sum(float x, int lanes) {
  for (int m = lanes >> 1; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
  return x;
}

template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void forward_heads(const NormRope& a, const View& in, const View& out, const void* weight, long long b, long long t,
                                              int h0, int h1, bool on, const Lane& ln, int lanes, const float2 (&c)[Half<T>::N], const float2 (&s)[Half<T>::N]) {
  constexpr int N = Half<T>::N;
  const Sides<T> w = weights_of<T, NEIGHBOURS>(weight, ln);
  float2 caw[N], sbw[N], saw[N], cbw[N];                   // a' = r (a caw - b sbw), b' = r (a saw + b cbw)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    caw[i] = mul_pair(c[i], w.a[i]);
    saw[i] = mul_pair(s[i], w.a[i]);
    cbw[i] = mul_pair(c[i], w.b[i]);
    sbw[i] = mul_pair(s[i], mul_pair(w.b[i], twice(-1.f)));
  }
  const T* x = reinterpret_cast<const T*>(in.p) + b * in.s0 + t * in.s2 + h0 * in.s1;
  T* y = reinterpret_cast<T*>(out.p) + b * out.s0 + t * out.s2 + h0 * out.s1;
  const float inv_d = 1.f / (float)a.d;
  for (int h = h0; h < h1; h += kAhead) {
    Pieces<T> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      raw[u].zero();
      if (on && h + u < h1) raw[u].load(x, ln);
      x += in.s1;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (h + u >= h1) break;
      Sides<T> v = raw[u].template get<NEIGHBOURS>();
      float2 q = mul_pair(v.a[0], v.a[0]);
      q = fma_pair(v.b[0], v.b[0], q);
#pragma unroll
      for (int i = 1; i < N; ++i) {
        q = fma_pair(v.a[i], v.a[i], q);
        q = fma_pair(v.b[i], v.b[i], q);
      }
      const float2 r = twice(rsqrtf(fmaf(row_sum(q.x + q.y, lanes), inv_d, a.eps)));
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 xa = mul_pair(v.a[i], r), xb = mul_pair(v.b[i], r);
        v.a[i] = fma_pair(xb, sbw[i], mul_pair(xa, caw[i]));
        v.b[i] = fma_pair(xa, saw[i], mul_pair(xb, cbw[i]));
      }
      if (on) {
        Pieces<T> o;
        o.template set<NEIGHBOURS>(v);
        o.store(y, ln);
      }
      y += out.s1;
    }
  }
}

__device__ __forceinline__ void share_turns(const NormRope& a, unsigned long long* turns) {
  for (int i = threadIdx.x; i < a.rot / 2; i += kThreads) turns[i] = a.turns[i];
  __syncthreads();
}

__device__ __forceinline__ long long position(const NormRope& a, long long b, long long t) {
  return a.positions != nullptr ? a.positions[b * a.ps0 + t * a.ps1] : a.pos_offset + t;
}

// grid: (groups of tokens, groups of heads_per heads of q and k together)
template <typename T, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, 4) norm_rope_kernel(const __grid_constant__ NormRope a, int lanes, int heads_per) {
  __shared__ unsigned long long turns[64];
  share_turns(a, turns);
  wait_for_kernels_ahead();
  const unsigned per = kThreads / lanes, tok = blockIdx.x * per + threadIdx.x / lanes;      // (at most 2^31 tokens)
  const bool on = tok < (unsigned long long)a.B * a.T;
  const unsigned b = on ? tok / (unsigned)a.T : 0, t = on ? tok - b * (unsigned)a.T : 0;
  const Lane ln = lane_of<T, NEIGHBOURS>(a, lanes);
  float2 c[Half<T>::N], s[Half<T>::N];
  turns_of<T, NEIGHBOURS>(turns, ln, position(a, b, t), c, s);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, a.Hq + a.Hk);
  if (h0 < a.Hq) forward_heads<T, NEIGHBOURS>(a, a.q, a.q_out, a.q_weight, b, t, h0, min(h1, a.Hq), on, ln, lanes, c, s);
  if (h1 > a.Hq) forward_heads<T, NEIGHBOURS>(a, a.k, a.k_out, a.k_weight, b, t, max(h0, a.Hq) - a.Hq, h1 - a.Hq, on, ln, lanes, c, s);
}

template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void backward_heads(const NormRope& a, const View& in, const View& grad, const View& out, const void* weight, long long b,
                                               long long t, int h0, int h1, bool on, const Lane& ln, int lanes, const float2 (&c)[Half<T>::N],
                                               const float2 (&s)[Half<T>::N], Sides<T>& dw) {
  constexpr int N = Half<T>::N;
  const Sides<T> w = weights_of<T, NEIGHBOURS>(weight, ln);
  const T* x = reinterpret_cast<const T*>(in.p) + b * in.s0 + t * in.s2 + h0 * in.s1;
  const T* g = reinterpret_cast<const T*>(grad.p) + b * grad.s0 + t * grad.s2 + h0 * grad.s1;
  T* y = reinterpret_cast<T*>(out.p) + b * out.s0 + t * out.s2 + h0 * out.s1;
  const float inv_d = 1.f / (float)a.d;
  for (int h = h0; h < h1; h += kBwdAhead) {
    Pieces<T> raw[kBwdAhead], graw[kBwdAhead];
#pragma unroll
    for (int u = 0; u < kBwdAhead; ++u) {
      raw[u].zero();
      graw[u].zero();
      if (on && h + u < h1) {
        raw[u].load(x, ln);
        graw[u].load(g, ln);
      }
      x += in.s1;
      g += grad.s1;
    }
#pragma unroll
    for (int u = 0; u < kBwdAhead; ++u) {
      if (h + u >= h1) break;
      Sides<T> v = raw[u].template get<NEIGHBOURS>(), z = graw[u].template get<NEIGHBOURS>();
      float2 q = twice(0.f), dot = twice(0.f);
#pragma unroll
      for (int i = 0; i < N; ++i) {                        // the turn back
        const float2 za = fma_pair(z.b[i], s[i], mul_pair(z.a[i], c[i]));
        z.b[i] = fma_pair(z.b[i], c[i], mul_pair(mul_pair(z.a[i], twice(-1.f)), s[i]));
        z.a[i] = za;
        q = fma_pair(v.a[i], v.a[i], q);
        q = fma_pair(v.b[i], v.b[i], q);
        dot = fma_pair(mul_pair(z.a[i], w.a[i]), v.a[i], dot);
        dot = fma_pair(mul_pair(z.b[i], w.b[i]), v.b[i], dot);
      }
      // (every lane takes part in the sums, also one without a token)
      const float square = row_sum(q.x + q.y, lanes), product = row_sum(dot.x + dot.y, lanes);
      const float rr = on ? rsqrtf(fmaf(square, inv_d, a.eps)) : 0.f;
      const float2 r = twice(rr), m = twice(-product * rr * rr * inv_d);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 xa = mul_pair(v.a[i], r), xb = mul_pair(v.b[i], r);
        dw.a[i] = fma_pair(z.a[i], xa, dw.a[i]);
        dw.b[i] = fma_pair(z.b[i], xb, dw.b[i]);
        v.a[i] = fma_pair(xa, m, mul_pair(mul_pair(z.a[i], w.a[i]), r));
        v.b[i] = fma_pair(xb, m, mul_pair(mul_pair(z.b[i], w.b[i]), r));
      }
      if (on) {
        Pieces<T> o;
        o.template set<NEIGHBOURS>(v);
        o.store(y, ln);
      }
      y += out.s1;
    }
  }
}

// Sums of the weights' gradients over the lanes and warps of a block: part[d].  Fixed order.
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void block_sum(const Sides<T>& dw, int lanes, const Lane& ln, int d, float* red, float* part) {
  constexpr int E = Half<T>::E, N = Half<T>::N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[4] = {dw.a[i].x, dw.a[i].y, dw.b[i].x, dw.b[i].y};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      for (int m = lanes; m < 32; m <<= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], m);
      // entry of side k / 2, number 2 i + k % 2 of this lane's
      const int j = 2 * i + (k & 1), e = NEIGHBOURS ? 2 * j + (k >> 1) : (k >> 1) * E + j;
      if (lane < lanes) red[warp * 128 + (e < E ? ln.e0 + e : ln.e1 + e - E)] = v[k];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < d; e += kThreads) {
    float sum = 0.f;
#pragma unroll
    for (int y = 0; y < kThreads / 32; ++y) sum += red[y * 128 + e];
    part[e] = sum;
  }
  __syncthreads();
}

// part: [blocks][2][d] (queries, keys), or null
template <typename T, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, 3) norm_rope_bwd_kernel(const __grid_constant__ NormRope a, int lanes, int heads_per, unsigned tok_groups,
                                                                    float* __restrict__ part) {
  __shared__ unsigned long long turns[64];
  __shared__ float red[kThreads / 32 * 128];
  share_turns(a, turns);
  wait_for_kernels_ahead();
  const unsigned per = kThreads / lanes;
  const Lane ln = lane_of<T, NEIGHBOURS>(a, lanes);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, a.Hq + a.Hk);
  Sides<T> dqw, dkw;
#pragma unroll
  for (int i = 0; i < Half<T>::N; ++i) dqw.a[i] = dqw.b[i] = dkw.a[i] = dkw.b[i] = twice(0.f);
  for (unsigned grp = blockIdx.x; grp < tok_groups; grp += gridDim.x) {
    const unsigned long long tok = (unsigned long long)grp * per + threadIdx.x / lanes;
    const bool on = tok < (unsigned long long)a.B * a.T;
    const unsigned b = on ? (unsigned)tok / (unsigned)a.T : 0, t = on ? (unsigned)tok - b * (unsigned)a.T : 0;
    float2 c[Half<T>::N], s[Half<T>::N];
    turns_of<T, NEIGHBOURS>(turns, ln, position(a, b, t), c, s);
    if (h0 < a.Hq) backward_heads<T, NEIGHBOURS>(a, a.q, a.q_out, a.dq, a.q_weight, b, t, h0, min(h1, a.Hq), on, ln, lanes, c, s, dqw);
    if (h1 > a.Hq)
      backward_heads<T, NEIGHBOURS>(a, a.k, a.k_out, a.dk, a.k_weight, b, t, max(h0, a.Hq) - a.Hq, h1 - a.Hq, on, ln, lanes, c, s, dkw);
  }
  if (part == nullptr) return;
  float* mine = part + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.d;
  block_sum<T, NEIGHBOURS>(dqw, lanes, ln, a.d, red, mine);
  block_sum<T, NEIGHBOURS>(dkw, lanes, ln, a.d, red, mine + a.d);
}

// Eight entries of a tensor's weights per block: the blocks' sums, 32 runs of them side by side, then the runs in order.
__global__ void __launch_bounds__(256) norm_rope_sum_kernel(const float* __restrict__ part, int blocks, int d, float* __restrict__ dq_weight,
                                                            float* __restrict__ dk_weight) {
  __shared__ float red[32][9];
  wait_for_kernels_ahead();
  float* to = blockIdx.x == 0 ? dq_weight : dk_weight;
  if (to == nullptr) return;
  const int i = threadIdx.x & 7, y = threadIdx.x >> 3, e = blockIdx.y * 8 + i;
  float sum = 0.f;
  for (int b = y; b < blocks; b += 8 * 32) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = b + u * 32 < blocks ? part[((size_t)(b + u * 32) * 2 + blockIdx.x) * d + e] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += v[u];
  }
  red[y][i] = sum;
  __syncthreads();
  if (y != 0) return;
#pragma unroll
  for (int k = 1; k < 32; ++k) sum += red[k][i];
  to[e] = sum;
}

struct RopeGrid {
  int lanes, heads_per;
  long long tok_groups;
  dim3 grid;
};
// Heads of a token in two blocks, or in more (down to `step` heads) while there are fewer blocks than fill the GPU. 
RopeGrid rope_grid(int B, int T, int H, int d, int elem, int step, bool backward) {
  RopeGrid g;
  g.lanes = d * elem / 16;
  const int per = kThreads / g.lanes;
  g.tok_groups = ((long long)B * T + per - 1) / per;
  g.heads_per = (H + 1) / 2 > step ? (H + 1) / 2 : step;
  while (g.heads_per > step && g.tok_groups * ((H + g.heads_per - 1) / g.heads_per) < kBlocks) g.heads_per = (g.heads_per + 1) / 2;
  const long long y = (H + g.heads_per - 1) / g.heads_per, most = backward ? (kBlocks + y - 1) / y : g.tok_groups;
  g.grid = dim3((unsigned)(g.tok_groups < most ? g.tok_groups : most), (unsigned)y);
  return g;
}

template <typename T> void forward(const NormRope& a, LaunchCtx& ctx) {
  const RopeGrid g = rope_grid(a.B, a.T, a.Hq + a.Hk, a.d, sizeof(T), 1, false);
  launch_after(ctx, a.interleaved ? norm_rope_kernel<T, true> : norm_rope_kernel<T, false>, g.grid, dim3(kThreads), 0, a, g.lanes, g.heads_per);
}

template <typename T> void backward(const NormRope& a, float* ws, LaunchCtx& ctx) {
  const RopeGrid g = rope_grid(a.B, a.T, a.Hq + a.Hk, a.d, sizeof(T), kBwdAhead, true);
  const bool sums = a.dq_weight != nullptr || a.dk_weight != nullptr;
  launch_after(ctx, a.interleaved ? norm_rope_bwd_kernel<T, true> : norm_rope_bwd_kernel<T, false>, g.grid, dim3(kThreads), 0, a, g.lanes, g.heads_per,
               (unsigned)g.tok_groups, sums ? ws : nullptr);
  if (sums) launch_after(ctx, norm_rope_sum_kernel, dim3(2, a.d / 8), dim3(256), 0, ws, (int)(g.grid.x * g.grid.y), a.d, a.dq_weight, a.dk_weight);
}

}  // namespace

void norm_rope_fwd(const NormRope& a, LaunchCtx& ctx) {
  if (a.dtype == KATA_F32) forward<float>(a, ctx);
  else forward<__nv_bfloat16>(a, ctx);
}

// (the larger of the two element types': the scratch depends on sizes alone)
size_t norm_rope_bwd_workspace_elems(int B, int T, int H, int d) {
  size_t blocks = 0;
  for (int elem = 2; elem <= 4; elem += 2) {
    const RopeGrid g = rope_grid(B, T, H, d, elem, kBwdAhead, true);
    if ((size_t)g.grid.x * g.grid.y > blocks) blocks = (size_t)g.grid.x * g.grid.y;
  }
  return blocks * 2 * d;
}

void norm_rope_bwd(const NormRope& a, float* ws, LaunchCtx& ctx) {
  if (a.dtype == KATA_F32) backward<float>(a, ws, ctx);
  else backward<__nv_bfloat16>(a, ws, ctx);
}

}  // namespace kata
