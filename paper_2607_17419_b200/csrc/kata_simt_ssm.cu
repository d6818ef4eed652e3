// Selective state space scan token by token in fp32 (every element type and size), and the sum over the segments of a head.
//   S <- a_t S + s_t k_t v_t^T,  o_t = S^T q_t + D v_t
// One CTA per head and segment of the tokens, the state in registers: a thread has one column and a quarter of the rows.  Tokens are
// staged 16 at a time (s_t folded into the keys), the next 16 on their way meanwhile; the four sums of an output meet in shared
// memory.  Bound by fp32 issue, three operations per state entry and token, where an SM has several CTAs, and by their latency where
// it has one.  Measured, fp32, n = d_v = 64, 128 tokens of a head: 13 and 17.6 us; 128 heads x 2000 tokens: 281 us.
// Few heads: the token axis is cut into segments.  Their own states (from zero) come first, ssm_prefix turns them into the states
// before the segments, and the second pass starts from those.
#include <cmath>

#include "kata_rows.cuh"
#include "kata_ssm.cuh"

namespace kata {
namespace {

constexpr int TB = 16;                 // tokens staged at a time
constexpr int RG = 4;                  // threads that share a column

template <typename T, int N, int DV, bool STATE>
__global__ void __launch_bounds__(DV * RG) simt_ssm_kernel(const __grid_constant__ Ssm a, const SsmPlan plan, float* __restrict__ ws) {
  constexpr int THREADS = DV * RG, R = N / RG, E = 16 / sizeof(T);
  constexpr int NQ = (TB * N / E + THREADS - 1) / THREADS, NV = (TB * DV / E + THREADS - 1) / THREADS;
  __shared__ __align__(16) float ks[TB][N], qs[STATE ? 1 : TB][N], vs[TB][DV], part[STATE ? 1 : TB][RG][DV];
  __shared__ float as[TB];
  wait_for_kernels_ahead();
  const int bh = blockIdx.x / plan.segments, seg = blockIdx.x % plan.segments;
  if (STATE && seg + 1 == plan.segments) return;
  const int b = bh / a.H, h = bh - b * a.H, g = h / (a.H / a.G), tid = threadIdx.x, col = tid % DV, rg = tid / DV;
  const int len = sequence_length(a.lengths, b, a.T);
  const int t0 = seg * plan.seg_tokens, t1 = min(t0 + plan.seg_tokens, a.T), live = min(t1, len);
  const T* kp = reinterpret_cast<const T*>(a.k.p) + b * a.k.s0 + g * a.k.s1;
  const T* qp = reinterpret_cast<const T*>(a.q.p) + b * a.q.s0 + g * a.q.s1;
  const T* vp = reinterpret_cast<const T*>(a.v.p) + b * a.v.s0 + h * a.v.s1;
  const T* dp = reinterpret_cast<const T*>(a.dt.p) + b * a.dt.s0 + h * a.dt.s1;
  T* op = reinterpret_cast<T*>(a.out.p) + b * a.out.s0 + h * a.out.s1;
  const float A = a.A[h], skip = a.D != nullptr ? a.D[h] : 0.f;
  constexpr size_t SE = (size_t)N * DV;
  float2 S[R / 2];                     // rows rg R + 2 r, + 1
  const float* init = STATE ? nullptr : plan.segments > 1 ? ws + ssm_slot(plan.segments, bh, seg) * SE : a.s_init != nullptr ? a.s_init + (size_t)bh * SE : nullptr;
#pragma unroll
  for (int r = 0; r < R / 2; ++r)
    S[r] = init != nullptr ? make_float2(init[(rg * R + 2 * r) * DV + col], init[(rg * R + 2 * r + 1) * DV + col]) : make_float2(0.f, 0.f);
  Entries<T, E> kr[NQ], qr[NQ], vr[NV];
  float dr = 0.f;
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int e = (tid + i * THREADS) * E, row = t + e / N;
      kr[i].zero();
      qr[i].zero();
      if (e < TB * N && row < live) {
        kr[i].load(kp + row * a.k.s2 + e % N);
        if (!STATE) qr[i].load(qp + row * a.q.s2 + e % N);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = (tid + i * THREADS) * E, row = t + e / DV;
      vr[i].zero();
      if (e < TB * DV && row < live) vr[i].load(vp + row * a.v.s2 + e % DV);
    }
    if (tid < TB && t + tid < live) dr = to_f32<T>(dp[(t + tid) * a.dt.s2]);
  };
  __shared__ float ss[TB];
  double decay = 0.0;                  // log of the decay over the segment, this thread's tokens
  if (t0 < live) fetch(t0);
  for (int t = t0; t < live; t += TB) {
    __syncthreads();
    if (tid < TB) {
      const float s = t + tid < live ? ssm_step_size(a, dr, h) : 0.f;
      ss[tid] = s;
      as[tid] = expf(s * A);
      if (STATE) decay += (double)s * A;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int e = (tid + i * THREADS) * E;
      if (e < TB * N) {
        float x[E];
        kr[i].get(x);
        const float s = ss[e / N];
#pragma unroll
        for (int j = 0; j < E; ++j) ks[e / N][e % N + j] = s * x[j];
        if (!STATE) {
          qr[i].get(x);
#pragma unroll
          for (int j = 0; j < E; ++j) qs[e / N][e % N + j] = x[j];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = (tid + i * THREADS) * E;
      if (e < TB * DV) {
        float x[E];
        vr[i].get(x);
#pragma unroll
        for (int j = 0; j < E; ++j) vs[e / DV][e % DV + j] = x[j];
      }
    }
    __syncthreads();
    if (t + TB < live) fetch(t + TB);
#pragma unroll(R <= 8 ? 8 : R <= 16 ? 4 : 2)
    for (int u = 0; u < TB; ++u) {
      const float2 v = make_float2(vs[u][col], vs[u][col]), d = make_float2(as[u], as[u]);
      float2 y = make_float2(0.f, 0.f);
#pragma unroll
      for (int r = 0; r < R / 2; r += 2) {
        const float4 k4 = *reinterpret_cast<const float4*>(&ks[u][rg * R + 2 * r]);
        S[r] = fma_pair(d, S[r], mul_pair(make_float2(k4.x, k4.y), v));
        S[r + 1] = fma_pair(d, S[r + 1], mul_pair(make_float2(k4.z, k4.w), v));
        if (!STATE) {
          const float4 q4 = *reinterpret_cast<const float4*>(&qs[u][rg * R + 2 * r]);
          y = fma_pair(make_float2(q4.x, q4.y), S[r], y);
          y = fma_pair(make_float2(q4.z, q4.w), S[r + 1], y);
        }
      }
      if (!STATE) part[u][rg][col] = y.x + y.y;
    }
    if (!STATE) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TB / RG; ++i) {
        const int u = i * RG + rg;
        if (t + u < live)
          op[(t + u) * a.out.s2 + col] = from_f32<T>(fmaf(skip, vs[u][col], (part[u][0][col] + part[u][1][col]) + (part[u][2][col] + part[u][3][col])));
      }
    }
  }
  if constexpr (STATE) {
    float* to = ws + ssm_slot(plan.segments, bh, seg + 1) * SE;
#pragma unroll
    for (int r = 0; r < R / 2; ++r) {
      to[(rg * R + 2 * r) * DV + col] = S[r].x;
      to[(rg * R + 2 * r + 1) * DV + col] = S[r].y;
    }
    if (tid < 32) {
      if (tid >= TB) decay = 0.0;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) decay += __shfl_xor_sync(0xffffffffu, decay, off);
      if (tid == 0) ws[(size_t)a.B * a.H * plan.segments * SE + ssm_slot(plan.segments, bh, seg)] = expf((float)decay);
    }
  } else {
    for (int t = max(live, t0) + rg; t < t1; t += RG) op[t * a.out.s2 + col] = from_f32<T>(0.f);
    if (a.s_final != nullptr && seg + 1 == plan.segments) {
#pragma unroll
      for (int r = 0; r < R / 2; ++r) {
        a.s_final[(size_t)bh * SE + (rg * R + 2 * r) * DV + col] = S[r].x;
        a.s_final[(size_t)bh * SE + (rg * R + 2 * r + 1) * DV + col] = S[r].y;
      }
    }
  }
}

// Slot j of a head: from the own state of segment j - 1 to the state before segment j (slot 0: the state handed in).  s_final: the
// state after the last segment, whose own state is in the slot behind.
__global__ void __launch_bounds__(128) ssm_prefix_kernel(float* __restrict__ ws, const float* s_init, float* s_final, int BH, int segments, int slots, int se) {
  wait_for_kernels_ahead();
  constexpr int U = 8;
  const int bh = blockIdx.y, e = blockIdx.x * 128 + threadIdx.x;           // (n d_v is a multiple of 128)
  float* s = ws + (size_t)bh * slots * se + e;
  const float* decay = ws + (size_t)BH * slots * se + (size_t)bh * slots;
  float cur = s_init != nullptr ? s_init[(size_t)bh * se + e] : 0.f;
  s[0] = cur;
  for (int j = 1; j < slots; j += U) {
    float own[U], d[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j + u < slots) {
        own[u] = s[(size_t)(j + u) * se];
        d[u] = decay[j + u - 1];
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j + u < slots) {
        cur = fmaf(d[u], cur, own[u]);
        if (j + u < segments) s[(size_t)(j + u) * se] = cur;
      }
  }
  if (s_final != nullptr) s_final[(size_t)bh * se + e] = cur;
}

template <typename T, int N, int DV> void launch(const Ssm& a, const SsmPlan& plan, float* ws, LaunchCtx& ctx) {
  const dim3 grid((unsigned)(a.B * a.H) * plan.segments);
  // A CTA that is resident early has to take the SM that is left: behind ssm_prefix, or another kernel of many CTAs, some SMs then get
  // several of these and others none.  (fp32, n = d_v = 64, 16 heads x 1000 tokens: 43.6 us early, 29.4 us not; 256 heads x 512 tokens: 154 and
  // 115.  Short calls gain a little by being there: 2 heads x 512, n = d_v = 16: 8.9 and 9.8, 16 heads x 40: 9.2 and 9.3.)
  const bool early = a.T <= 64;
  if (plan.segments > 1) {
    launch_when(early, ctx, simt_ssm_kernel<T, N, DV, true>, grid, dim3(DV * RG), 0, a, plan, ws);
    ssm_prefix(a, plan, plan.segments, ws, ctx);
  }
  launch_when(early, ctx, simt_ssm_kernel<T, N, DV, false>, grid, dim3(DV * RG), 0, a, plan, ws);
}

template <typename T, int N> void by_width(const Ssm& a, const SsmPlan& plan, float* ws, LaunchCtx& ctx) {
  if (a.d == 16) launch<T, N, 16>(a, plan, ws, ctx);
  else if (a.d == 32) launch<T, N, 32>(a, plan, ws, ctx);
  else launch<T, N, 64>(a, plan, ws, ctx);
}

template <typename T> void by_rows(const Ssm& a, const SsmPlan& plan, float* ws, LaunchCtx& ctx) {
  if (a.n == 16) by_width<T, 16>(a, plan, ws, ctx);
  else if (a.n == 32) by_width<T, 32>(a, plan, ws, ctx);
  else if (a.n == 64) by_width<T, 64>(a, plan, ws, ctx);
  else by_width<T, 128>(a, plan, ws, ctx);
}

}  // namespace

// Segments of whole tiles (128 tokens on the tensor cores, else 32) and how long a pass takes by the rates measured here: a tile of
// the outputs and one of the states, in us, times the CTAs that an SM has in a row.  On the tensor cores an SM has one CTA; of the
// token by token kernel it runs 1.25 of 256 threads (2.5 of 128, 5 of 64) as fast as one.  Several segments, and a final state on the
// tensor cores, take the pass of the states too.  The smallest sum wins; more CTAs than eight per SM never did.  Measured, us with one
// segment / two / this rule's: fp32, n = d_v = 64, 16 heads x 1000 tokens: 142 / 118 / 29; bf16, n = d_v = 16, 16 heads x 16384: 1320 /
// 1035 / 58; fp32, n = d_v = 64, 128 heads x 2000 (the rule stays with one): 281 / 350 / 281.
// The sequences of a padded batch count as if they filled it: their lengths are on the device.  (Counted as half full on average, with a
// final state, us with lengths uniform / all full / one long among short, against this: 4 x 16 heads x 3001, n = 128: 54 to 61 / 86 / 46
// against 62 / 63 / 61; 2 x 16 heads x 3001, n = 64: 30 to 43 / 42 / 28 against 30 / 30 / 30.)
SsmPlan ssm_plan(int BH, int T, int n, int d, bool tensor, bool final_state) {
  const int tile = tensor ? 128 : 32, tiles = (T + tile - 1) / tile;
  const double out_us = tensor ? 1.85 : 2.0 + 0.039 * n, state_us = tensor ? 0.75 : 0.6 * out_us;
  const double together = tensor ? 1.0 : 80.0 / d;
  const long long most = kPlanSMs * (tensor ? 2LL : 8LL);
  SsmPlan best{1, tiles * tile};
  double best_us = 0.0;
  for (int want = 1; want <= tiles && (want == 1 || (long long)BH * (want - 1) < most); ++want) {
    const int per = (tiles + want - 1) / want, segments = (tiles + per - 1) / per;
    const bool states = segments > 1 || (tensor && final_state);
    const long long row = ((long long)BH * segments + kPlanSMs - 1) / kPlanSMs;
    const double us = (row > together ? row / together : 1.0) * per * (out_us + (states ? state_us : 0.0)) +
                      (states ? (tensor ? 8.0 + 0.1 * segments : 3.0 + 0.07 * segments) : 0.0);
    if (want == 1 || us < best_us) {
      best_us = us;
      best = SsmPlan{segments, per * tile};
    }
  }
  return best;
}

size_t ssm_workspace_bytes(int BH, int n, int d, int slots) { return (size_t)BH * slots * ((size_t)n * d + 1) * sizeof(float); }

void ssm_prefix(const Ssm& a, const SsmPlan& plan, int slots, float* ws, LaunchCtx& ctx) {
  launch_after(ctx, ssm_prefix_kernel, dim3(a.n * a.d / 128, a.B * a.H), dim3(128), 0, ws, a.s_init, slots > plan.segments ? a.s_final : nullptr, a.B * a.H,
               plan.segments, slots, a.n * a.d);
}

void simt_ssm(const Ssm& a, const SsmPlan& plan, float* ws, LaunchCtx& ctx) {
  if (a.dtype == KATA_F32) by_rows<float>(a, plan, ws, ctx);
  else by_rows<__nv_bfloat16>(a, plan, ws, ctx);
}

}  // namespace kata
