// Norm of query and key rows by their root mean square and rotation by their positions, and the backward of both:
//   y = R_p (w * x r),  r = 1 / sqrt(mean(x^2) + eps)
//   u = R_p^T dy,  dw = sum u * x r,  dx = r (u * w - x r mean(u * w * x r))
// HBM-bound: every row is read and written once (backward: two reads, one write).  A row is held by d / (16 bytes) neighbouring
// lanes, 16 bytes each.  The turn of a pair depends on the token and not on the head, so the lanes of a token form their sines
// once and walk the heads with them.  An entry of the result is r (x c + x' s) with x' the other entry of its pair, c = cos w and
// s = -+ sin w': the pair's raw 16 bytes come from their lane by four shuffles.
// Angles: position times a 64-bit fraction of a turn, in wrapping integers: no rounding grows with the position.
#include "kata_rows.cuh"

namespace kata {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;                // heads in flight
constexpr int kMaxBwdBlocks = 4 * kPlanSMs;

// cos and +-sin of this lane's entries at a position (the sign of the entry's side of the pair: y = x cos + x' sin).
template <int E, bool NEIGHBOURS>
__device__ __forceinline__ void turns_of(const NormRope& a, const unsigned long long* turns, int e0, long long pos, float (&c)[E], float (&s)[E]) {
  const int half = a.rot / 2;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const int i = e0 + j;
    c[j] = 1.f;
    s[j] = 0.f;
    if (i < a.rot) {
      if (NEIGHBOURS && (j & 1)) {
        c[j] = c[j - 1];
        s[j] = -s[j - 1];
      } else {
        const int f = NEIGHBOURS ? i / 2 : (i < half ? i : i - half);
        const unsigned long long turn = (unsigned long long)pos * turns[f];
        float sn;
        sincospif((float)(int)(turn >> 32) * 4.656612873077392578125e-10f, &sn, &c[j]);     // half turns in [-1, 1)
        s[j] = NEIGHBOURS || i < half ? -sn : sn;
      }
    }
  }
}

// The raw entries of the other side of the pairs.
template <typename T, int E, bool NEIGHBOURS>
__device__ __forceinline__ void partner(const Entries<T, E>& x, int src, float (&out)[E]) {
  if (NEIGHBOURS) {
    float v[E];
    x.get(v);
#pragma unroll
    for (int j = 0; j < E; ++j) out[j] = v[j ^ 1];
  } else {
    Entries<T, E> y;
    y.raw.x = __shfl_sync(0xffffffffu, x.raw.x, src);
    y.raw.y = __shfl_sync(0xffffffffu, x.raw.y, src);
    y.raw.z = __shfl_sync(0xffffffffu, x.raw.z, src);
    y.raw.w = __shfl_sync(0xffffffffu, x.raw.w, src);
    y.get(out);
  }
}

struct Lane {
  int e0, src;                            // first entry, lane of the other side of its pairs
};
template <int E>
__device__ __forceinline__ Lane lane_of(const NormRope& a, int lanes) {
  const int lane = threadIdx.x & 31, l = lane & (lanes - 1), half = a.rot / 2 / E;        // (of half-split pairs)
  Lane r;
  r.e0 = l * E;
  r.src = l < half ? lane + half : l < 2 * half ? lane - half : lane;
  return r;
}

template <typename T, int E>
__device__ __forceinline__ void load_weight(const void* w, int e0, float (&out)[E]) {
#pragma unroll
  for (int j = 0; j < E; ++j) out[j] = w != nullptr ? to_f32<T>(static_cast<const T*>(w)[e0 + j]) : 1.f;
}

template <typename T, int E, bool NEIGHBOURS>
__device__ __forceinline__ void forward_heads(const NormRope& a, const View& in, const View& out, const void* weight, long long b, long long t,
                                              int h0, int h1, bool on, const Lane& ln, int lanes, const float (&c)[E], const float (&s)[E]) {
  float cw[E], sw[E], w[E];
  load_weight<T, E>(weight, ln.e0, w);
  const int half = a.rot / 2, e1 = ln.e0 < half ? ln.e0 + half : ln.e0 - half;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    cw[j] = c[j] * w[j];
    sw[j] = 0.f;
    if (ln.e0 + j < a.rot) sw[j] = s[j] * (NEIGHBOURS ? w[j ^ 1] : weight != nullptr ? to_f32<T>(static_cast<const T*>(weight)[e1 + j]) : 1.f);
  }
  const T* x = reinterpret_cast<const T*>(in.p) + b * in.s0 + t * in.s2 + ln.e0;
  T* y = reinterpret_cast<T*>(out.p) + b * out.s0 + t * out.s2 + ln.e0;
  const float inv_d = 1.f / (float)a.d;
  for (int h = h0; h < h1; h += kAhead) {
    Entries<T, E> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      raw[u].zero();
      if (on && h + u < h1) raw[u].load(x + (long long)(h + u) * in.s1);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (h + u >= h1) break;
      float v[E], o[E], ss = 0.f;
      raw[u].get(v);
      partner<T, E, NEIGHBOURS>(raw[u], ln.src, o);
#pragma unroll
      for (int j = 0; j < E; ++j) ss = fmaf(v[j], v[j], ss);
      for (int m = lanes >> 1; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
      const float r = rsqrtf(fmaf(ss, inv_d, a.eps));
#pragma unroll
      for (int j = 0; j < E; ++j) v[j] = r * fmaf(o[j], sw[j], v[j] * cw[j]);
      if (on) {
        Entries<T, E> st;
        st.set(v);
        st.store(y + (long long)(h + u) * out.s1);
      }
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
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ NormRope a, int lanes, int heads_per) {
  constexpr int E = 16 / sizeof(T);
  __shared__ unsigned long long turns[64];
  share_turns(a, turns);
  wait_for_kernels_ahead();
  const int per = kThreads / lanes;
  const long long tok = (long long)blockIdx.x * per + threadIdx.x / lanes;
  const bool on = tok < (long long)a.B * a.T;
  const long long b = on ? tok / a.T : 0, t = on ? tok - b * a.T : 0;
  const Lane ln = lane_of<E>(a, lanes);
  float c[E], s[E];
  turns_of<E, NEIGHBOURS>(a, turns, ln.e0, position(a, b, t), c, s);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, a.Hq + a.Hk);
  if (h0 < a.Hq) forward_heads<T, E, NEIGHBOURS>(a, a.q, a.q_out, a.q_weight, b, t, h0, min(h1, a.Hq), on, ln, lanes, c, s);
  if (h1 > a.Hq) forward_heads<T, E, NEIGHBOURS>(a, a.k, a.k_out, a.k_weight, b, t, max(h0, a.Hq) - a.Hq, h1 - a.Hq, on, ln, lanes, c, s);
}

template <typename T, int E, bool NEIGHBOURS>
__device__ __forceinline__ void backward_heads(const NormRope& a, const View& in, const View& grad, const View& out, const void* weight, long long b,
                                               long long t, int h0, int h1, bool on, const Lane& ln, int lanes, const float (&c)[E],
                                               const float (&s)[E], float (&dw)[E]) {
  float w[E];
  load_weight<T, E>(weight, ln.e0, w);
  const T* x = reinterpret_cast<const T*>(in.p) + b * in.s0 + t * in.s2 + ln.e0;
  const T* g = reinterpret_cast<const T*>(grad.p) + b * grad.s0 + t * grad.s2 + ln.e0;
  T* y = reinterpret_cast<T*>(out.p) + b * out.s0 + t * out.s2 + ln.e0;
  const float inv_d = 1.f / (float)a.d;
  constexpr int AHEAD = kAhead / 2;
  for (int h = h0; h < h1; h += AHEAD) {
    Entries<T, E> raw[AHEAD], graw[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      raw[u].zero();
      graw[u].zero();
      if (on && h + u < h1) {
        raw[u].load(x + (long long)(h + u) * in.s1);
        graw[u].load(g + (long long)(h + u) * grad.s1);
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (h + u >= h1) break;
      float v[E], z[E], o[E], ss = 0.f, dot = 0.f;
      raw[u].get(v);
      graw[u].get(z);
      partner<T, E, NEIGHBOURS>(graw[u], ln.src, o);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        z[j] = fmaf(-s[j], o[j], z[j] * c[j]);              // the turn back
        ss = fmaf(v[j], v[j], ss);
        dot = fmaf(z[j] * w[j], v[j], dot);
      }
      for (int m = lanes >> 1; m > 0; m >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, m);
        dot += __shfl_xor_sync(0xffffffffu, dot, m);
      }
      const float r = on ? rsqrtf(fmaf(ss, inv_d, a.eps)) : 0.f;
      const float m = dot * r * r * inv_d;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        dw[j] = fmaf(z[j], v[j] * r, dw[j]);
        v[j] = r * fmaf(-m, v[j], z[j] * w[j]);
      }
      if (on) {
        Entries<T, E> st;
        st.set(v);
        st.store(y + (long long)(h + u) * out.s1);
      }
    }
  }
}

// Sums of the weights' gradients over the lanes and warps of a block: part[d].  Fixed order.
template <int E>
__device__ __forceinline__ void block_sum(float (&dw)[E], int lanes, int e0, int d, float* red, float* part) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < E; ++j)
    for (int m = lanes; m < 32; m <<= 1) dw[j] += __shfl_xor_sync(0xffffffffu, dw[j], m);
  if (lane < lanes)
#pragma unroll
    for (int j = 0; j < E; ++j) red[warp * 128 + e0 + j] = dw[j];
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
__global__ void __launch_bounds__(kThreads) norm_rope_bwd_kernel(const __grid_constant__ NormRope a, int lanes, int heads_per, long long tok_groups,
                                                                 float* __restrict__ part) {
  constexpr int E = 16 / sizeof(T);
  __shared__ unsigned long long turns[64];
  __shared__ float red[kThreads / 32 * 128];
  share_turns(a, turns);
  wait_for_kernels_ahead();
  const int per = kThreads / lanes;
  const Lane ln = lane_of<E>(a, lanes);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, a.Hq + a.Hk);
  float dqw[E], dkw[E];
#pragma unroll
  for (int j = 0; j < E; ++j) dqw[j] = dkw[j] = 0.f;
  for (long long grp = blockIdx.x; grp < tok_groups; grp += gridDim.x) {
    const long long tok = grp * per + threadIdx.x / lanes;
    const bool on = tok < (long long)a.B * a.T;
    const long long b = on ? tok / a.T : 0, t = on ? tok - b * a.T : 0;
    float c[E], s[E];
    turns_of<E, NEIGHBOURS>(a, turns, ln.e0, position(a, b, t), c, s);
    if (h0 < a.Hq) backward_heads<T, E, NEIGHBOURS>(a, a.q, a.q_out, a.dq, a.q_weight, b, t, h0, min(h1, a.Hq), on, ln, lanes, c, s, dqw);
    if (h1 > a.Hq)
      backward_heads<T, E, NEIGHBOURS>(a, a.k, a.k_out, a.dk, a.k_weight, b, t, max(h0, a.Hq) - a.Hq, h1 - a.Hq, on, ln, lanes, c, s, dkw);
  }
  if (part == nullptr) return;
  float* mine = part + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.d;
  block_sum<E>(dqw, lanes, ln.e0, a.d, red, mine);
  block_sum<E>(dkw, lanes, ln.e0, a.d, red, mine + a.d);
}

// One block per tensor: the blocks' sums, 1024 / d runs of them side by side, then the runs in order.
__global__ void __launch_bounds__(1024) norm_rope_sum_kernel(const float* __restrict__ part, int blocks, int d, float* __restrict__ dq_weight,
                                                             float* __restrict__ dk_weight) {
  __shared__ float red[1024];
  wait_for_kernels_ahead();
  float* to = blockIdx.x == 0 ? dq_weight : dk_weight;
  if (to == nullptr) return;
  const int e = threadIdx.x % d, y = threadIdx.x / d, ny = 1024 / d;
  float sum = 0.f;
  for (int b = y; b < blocks; b += ny) sum += part[((size_t)b * 2 + blockIdx.x) * d + e];
  red[threadIdx.x] = sum;
  __syncthreads();
  if (y != 0) return;
  for (int i = 1; i < ny; ++i) sum += red[i * d + e];
  to[e] = sum;
}

struct RopeGrid {
  int lanes, heads_per;
  long long tok_groups;
  dim3 grid;
};
// All heads of a token in one block, or fewer (down to one step of the loop) while there are fewer blocks than fill the GPU.
RopeGrid rope_grid(int B, int T, int H, int d, int elem, int step, long long max_x) {
  RopeGrid g;
  g.lanes = d * elem / 16;
  const int per = kThreads / g.lanes;
  g.tok_groups = ((long long)B * T + per - 1) / per;
  long long x = g.tok_groups < max_x ? g.tok_groups : max_x;
  g.heads_per = H;
  while (g.heads_per > step && x * ((H + g.heads_per - 1) / g.heads_per) < 4 * kPlanSMs) g.heads_per = (g.heads_per + 1) / 2;
  g.grid = dim3((unsigned)x, (unsigned)((H + g.heads_per - 1) / g.heads_per));
  return g;
}
constexpr int kBwdStep = kAhead / 2;

template <typename T> void forward(const NormRope& a, LaunchCtx& ctx) {
  const RopeGrid g = rope_grid(a.B, a.T, a.Hq + a.Hk, a.d, sizeof(T), 1, (1LL << 31) - 1);
  launch_after(ctx, a.interleaved ? norm_rope_kernel<T, true> : norm_rope_kernel<T, false>, g.grid, dim3(kThreads), 0, a, g.lanes, g.heads_per);
}

template <typename T> void backward(const NormRope& a, float* ws, LaunchCtx& ctx) {
  const RopeGrid g = rope_grid(a.B, a.T, a.Hq + a.Hk, a.d, sizeof(T), kBwdStep, kMaxBwdBlocks);
  const bool sums = a.dq_weight != nullptr || a.dk_weight != nullptr;
  launch_after(ctx, a.interleaved ? norm_rope_bwd_kernel<T, true> : norm_rope_bwd_kernel<T, false>, g.grid, dim3(kThreads), 0, a, g.lanes, g.heads_per,
               g.tok_groups, sums ? ws : nullptr);
  if (sums) launch_after(ctx, norm_rope_sum_kernel, dim3(2), dim3(1024), 0, ws, (int)(g.grid.x * g.grid.y), a.d, a.dq_weight, a.dk_weight);
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
    const RopeGrid g = rope_grid(B, T, H, d, elem, kBwdStep, kMaxBwdBlocks);
    if ((size_t)g.grid.x * g.grid.y > blocks) blocks = (size_t)g.grid.x * g.grid.y;
  }
  return blocks * 2 * d;
}

void norm_rope_bwd(const NormRope& a, float* ws, LaunchCtx& ctx) {
  if (a.dtype == KATA_F32) backward<float>(a, ws, ctx);
  else backward<__nv_bfloat16>(a, ws, ctx);
}

}  // namespace kata
