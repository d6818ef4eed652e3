// One token of the selective state space scan for every head (the decode step):
//   S <- a S + s k v^T,  out = S^T q + D v,  s = dt + bias (or log(1 + e^that)),  a = e^(s A)
// HBM-bound: the fp32 state [n][d_v] of a head is read and written once.  Columns of the state do not meet one another, so a CTA
// takes all rows of some columns and no partial sums leave it: one launch, no scratch.  A thread holds four neighbouring columns
// of every RG-th row, all of them loaded before the first is used; the sums over the rows go through shuffles and shared memory.
// Measured: 2048 heads, n = 128, d_v = 64, bf16: 22.1 us for 135 MB, 6.1 TB/s (states larger than L2); 16 heads, n = 64: 2.0 us, a launch
// and one round trip to memory.
#include "kata_rows.cuh"
#include "kata_ssm.cuh"

namespace kata {
namespace {

template <typename T, int N, int DV, int COLS>
struct StepShape {
  static constexpr int TC = COLS / 4;                                 // threads along a row
  static constexpr int RG = (256 / TC) < (N / 2) ? (256 / TC) : (N / 2);
  static constexpr int THREADS = TC * RG, R = N / RG, WARPS = THREADS / 32;
};

template <typename T, int N, int DV, int COLS>
__global__ void __launch_bounds__(StepShape<T, N, DV, COLS>::THREADS) ssm_step_kernel(const __grid_constant__ Ssm a) {
  typedef StepShape<T, N, DV, COLS> Sh;
  constexpr int TC = Sh::TC, RG = Sh::RG, R = Sh::R, WARPS = Sh::WARPS;
  static_assert(Sh::THREADS >= 32 && Sh::THREADS % 32 == 0 && R * RG == N && TC <= 32, "shape");
  __shared__ float4 red[WARPS][TC];
  const int bh = blockIdx.x, b = bh / a.H, h = bh - b * a.H, g = h / (a.H / a.G);
  const int tc = threadIdx.x % TC, rg = threadIdx.x / TC, col = blockIdx.y * COLS + tc * 4;
  wait_for_kernels_ahead();
  float4* S = reinterpret_cast<float4*>(a.s_final + ((size_t)bh * N) * DV + col);
  float4 st[R];
#pragma unroll
  for (int r = 0; r < R; ++r) st[r] = S[(size_t)(r * RG + rg) * (DV / 4)];
  const T* kp = reinterpret_cast<const T*>(a.k.p) + b * a.k.s0 + g * a.k.s1;
  const T* qp = reinterpret_cast<const T*>(a.q.p) + b * a.q.s0 + g * a.q.s1;
  Entries<T, 4> vr;
  vr.load(reinterpret_cast<const T*>(a.v.p) + b * a.v.s0 + h * a.v.s1 + col);
  float kk[R], qq[R], v[4];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    kk[r] = to_f32<T>(kp[r * RG + rg]);
    qq[r] = to_f32<T>(qp[r * RG + rg]);
  }
  const float s = ssm_step_size(a, to_f32<T>(reinterpret_cast<const T*>(a.dt.p)[b * a.dt.s0 + h * a.dt.s1]), h);
  const float decay = expf(s * a.A[h]);
  vr.get(v);
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float kx = s * kk[r];
    st[r].x = fmaf(kx, v[0], decay * st[r].x);
    st[r].y = fmaf(kx, v[1], decay * st[r].y);
    st[r].z = fmaf(kx, v[2], decay * st[r].z);
    st[r].w = fmaf(kx, v[3], decay * st[r].w);
    S[(size_t)(r * RG + rg) * (DV / 4)] = st[r];
    y.x = fmaf(qq[r], st[r].x, y.x);
    y.y = fmaf(qq[r], st[r].y, y.y);
    y.z = fmaf(qq[r], st[r].z, y.z);
    y.w = fmaf(qq[r], st[r].w, y.w);
  }
#pragma unroll
  for (int off = TC; off < 32; off <<= 1) {
    y.x += __shfl_xor_sync(0xffffffffu, y.x, off);
    y.y += __shfl_xor_sync(0xffffffffu, y.y, off);
    y.z += __shfl_xor_sync(0xffffffffu, y.z, off);
    y.w += __shfl_xor_sync(0xffffffffu, y.w, off);
  }
  if ((threadIdx.x & 31) < TC) red[threadIdx.x >> 5][tc] = y;
  __syncthreads();
  if (threadIdx.x >= TC) return;
  y = red[0][tc];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) {
    const float4 o = red[w][tc];
    y.x += o.x;
    y.y += o.y;
    y.z += o.z;
    y.w += o.w;
  }
  const float skip = a.D != nullptr ? a.D[h] : 0.f;
  const float out[4] = {fmaf(skip, v[0], y.x), fmaf(skip, v[1], y.y), fmaf(skip, v[2], y.z), fmaf(skip, v[3], y.w)};
  Entries<T, 4> e;
  e.set(out);
  e.store(reinterpret_cast<T*>(a.out.p) + b * a.out.s0 + h * a.out.s1 + col);
}

template <typename T, int N, int DV, int COLS>
void launch(const Ssm& a, LaunchCtx& ctx) {
  launch_after(ctx, ssm_step_kernel<T, N, DV, COLS>, dim3(a.B * a.H, DV / COLS), dim3(StepShape<T, N, DV, COLS>::THREADS), 0, a);
}

template <typename T, int N> void by_width(const Ssm& a, LaunchCtx& ctx) {
  // 16 columns a CTA while that leaves no SM with more than two.  Measured, us, 16 columns / a whole row, n = d_v = 64: 16 heads 2.02 /
  // 2.15, 64 heads 2.23 / 2.31, 128 heads 2.56 / 2.37; n = 128, 2048 heads: 28.3 / 22.1.
  const bool few = (long long)a.B * a.H * (a.d / 16) <= 2 * kPlanSMs;
  if (a.d == 16) launch<T, N, 16, 16>(a, ctx);
  else if (a.d == 32) few ? launch<T, N, 32, 16>(a, ctx) : launch<T, N, 32, 32>(a, ctx);
  else few ? launch<T, N, 64, 16>(a, ctx) : launch<T, N, 64, 64>(a, ctx);
}

template <typename T> void by_rows(const Ssm& a, LaunchCtx& ctx) {
  if (a.n == 16) by_width<T, 16>(a, ctx);
  else if (a.n == 32) by_width<T, 32>(a, ctx);
  else if (a.n == 64) by_width<T, 64>(a, ctx);
  else by_width<T, 128>(a, ctx);
}

}  // namespace

void ssm_step(const Ssm& a, LaunchCtx& ctx) {
  if (a.dtype == KATA_F32) by_rows<float>(a, ctx);
  else by_rows<__nv_bfloat16>(a, ctx);
}

}  // namespace kata
