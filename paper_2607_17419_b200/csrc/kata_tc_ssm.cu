// Selective state space scan on the Blackwell tensor cores: bf16, n = 64 or 128 state rows, d_v = 64.
//   S_t = a_t S_{t-1} + s_t k_t v_t^T,  o_t = S_t^T q_t + D v_t,  a_t = 2^(l_t), l_t = s_t A log2(e)
// in tiles of 128 tokens, c_t the sum of l up to token t of the tile:
//   out    O = [(Q K^T) o W] V + diag(2^c) Q S + D V,  W[t,i] = 2^(c_t - c_i) s_i for i <= t
//   state  S <- 2^(c_127) S + K^T diag(2^(c_127 - c_i) s_i) V
//
// tc_ssm_out_kernel: a CTA has one head and a segment of its tokens and walks the tiles.  Scores come from the tensor cores,
// builder warps weigh them in registers and put them back into TMEM as the bf16 A operand of the product with V.  Nothing but
// S ties the tiles together: its fp32 entries stay in TMEM, where four warps add the tile's own state (a product of
// its own, from V scaled and rounded to bf16) and leave a bf16 copy in shared memory for the next tile's Q S.
// The weights of a 32 x 32 block are a row factor times a column factor, taken at the start of the rows' block: below the diagonal
// both are at most s_i; on the diagonal they are taken at half of the block's decay, and only blocks that decay by more than 2^-240 in
// their 32 tokens, or whose step sizes take such a factor out of fp32's range, take an exponential per entry instead.  So a tile takes
// a few exponentials per token and two products per score.
// tc_ssm_state_kernel: the segments' own states (several segments, or a final state wanted).  For a final state they are exact to
// fp32: the scaled V goes in as three bf16 terms (24 bits), the small ones first; every tile's product is added in registers.
//
// Warps.  Out (768 threads): 0 decays; 1 issues Q K^T and Q S, 2 the tile's state and the product with V; 3 TMA loads;
// 4-7 state; 8-15 weights and 16-23 scaled V and epilogue, two warps per TMEM lane quadrant.  State (512): 0 loads, 1 issues, 2, 3 decays, 4-7
// state, 8-15 scaled V.  A warp reaches the next wait of its job long before the others are done with theirs, so a tile takes the longest
// job and not their sum.  The jobs' loops are written once each and kept short: sixteen warps in unlike code of some thousand instructions
// each waited for instructions most of the time (8 x 16 heads x 4096 tokens 135 us).
// Measured (n = 64): 8 x 16 heads x 4096 tokens 59.9 us (144 MB: 22 us at the copy bandwidth; 3500 cycles a tile); 16 heads x 131072, in
// segments with the state kernel before: 294 us (88 us).  Bound by instructions: a tile takes 8400 of the warps', two thirds of the issue
// slots with six warps a scheduler; the tensor cores and the memory wait.  Not kept: results in two buffers with weights in columns of
// their own (65 us), an issuing warp for each chain (66 us), scaling V in bf16 pairs (59 us, as then without).
// All waits are bounded; a warp that has TMEM to read goes on only where all its lanes saw the barrier.
#include <cuda.h>

#include "kata_rows.cuh"
#include "kata_ssm.cuh"
#include "kata_tmap.cuh"
#include "kata_umma.cuh"

namespace kata {
namespace {

using namespace umma;

constexpr int CT = 128;                          // tokens per tile
constexpr int DV = 64;
constexpr int kOutThreads = 768, kStateThreads = 512;
constexpr int W_STATE0 = 4, W_WEIGHT0 = 8, W_OUT0 = 16;
constexpr uint32_t HALF = 16384;                 // 128 rows of 64 bf16 entries, 128B swizzle
constexpr int NSLOT = 4;                         // tiles whose decays are held

// Decays of a tile, c_t counted from the start of the token's block of 32.
struct Decays {
  float row[CT];                                 // 2^(c_t)
  float tail[CT];                                // 2^(c at the end of the block - c_t) s_t
  float inv[CT];                                 // 2^(m - c_t) s_t, m half of c at the end of the block
  float left[CT];                                // 2^(c at the end of the tile - c_t) s_t
  float rel[CT], step[CT];                       // c_t, s_t
  float before[4];                               // 2^(c from the start of the tile to block b)
  float between[4][4];                           // [r][b]: 2^(c from the end of block b to the start of block r), b < r
  float total;                                   // 2^(c of the whole tile)
  float half[4];                                 // m
  float pad[3];
};

template <int N, int STATE> struct Shape {         // STATE: terms of the scaled V in the state kernel; 0: the out kernel
  static constexpr int HALVES = N / 64;                                        // 64-column halves of a q or k tile
  static constexpr uint32_t K_OFF = STATE ? 0 : HALVES * HALF, V_OFF = K_OFF + HALVES * HALF;
  static constexpr uint32_t STAGE = V_OFF + HALF;
  static constexpr int NST = N == 64 ? 3 : 2;
  static constexpr int TERMS = STATE ? STATE : 1;
  static constexpr int XB = !STATE && N == 128 ? 1 : 2;                        // buffers of scaled V
  static constexpr uint32_t OFF_X = NST * STAGE;
  static constexpr uint32_t OFF_S = OFF_X + XB * TERMS * HALF;                 // [N][64] bf16
  static constexpr uint32_t OFF_OUT = OFF_S + (STATE ? 0 : N * 128);           // 8 warps x 32 rows of 64 bytes
  static constexpr uint32_t OFF_DEC = OFF_OUT + (STATE ? 0 : HALF);
  static constexpr uint32_t OFF_BAR = OFF_DEC + NSLOT * sizeof(Decays);
  static constexpr uint32_t SMEM = OFF_BAR + 512 + 1024;
};
static_assert(Shape<128, 0>::SMEM <= 232448 && Shape<64, 0>::SMEM <= 232448, "shared memory");
static_assert(Shape<128, 3>::SMEM <= 232448 && Shape<64, 3>::SMEM <= 232448, "shared memory");
static_assert(Shape<64, 0>::SMEM > 116 * 1024 && Shape<64, 1>::SMEM > 116 * 1024, "one CTA per SM is assumed (it takes all of TMEM)");

constexpr uint32_t COL_P = 0;                    // 2 x 128: scores; the bf16 weights overwrite columns [0,32) and [64,96) of a buffer
constexpr uint32_t COL_Y = 256, COL_R = 320;     // product with V, Q S
constexpr uint32_t COL_SL = 384, COL_S = 448;    // own state of a tile, state (state kernel: 2 x 64, own states)
constexpr uint32_t TMEM_COLS = 512;

// Every barrier's phases are seen in order by all that wait for it before the next can complete (see the notes at the waits).
enum {
  BAR_FULL = 0,        // [3] tile landed
  BAR_EMPTY = 3,       // [3] out: Q S and product with V done (2 commits), V read (8 warps); state: the state product done
  BAR_DEC_FULL = 6,    // [4] decays in place (32)
  BAR_DEC_EMPTY = 10,  // [4] decays read (one arrival per reading warp)
  BAR_S_FULL = 14,     // [2] scores in TMEM
  BAR_P_FULL = 16,     // [2] weights in TMEM (256)
  BAR_P_EMPTY = 18,    // [2] weights consumed
  BAR_O_FULL = 20,     // both products of a tile done (2 commits)
  BAR_O_EMPTY = 21,    // results read (256)
  BAR_X_FULL = 22,     // [2] scaled V in place (its warps' threads)
  BAR_X_EMPTY = 24,    // [2] consumed
  BAR_SL_FULL = 26,    // [2] own state of a tile in TMEM
  BAR_SL_EMPTY = 28,   // [2] read (128)
  BAR_ST = 30,         // bf16 state for the next tile in place (128)
  BAR_R_DONE = 31,     // Q S done: the bf16 state may be overwritten
  BAR_DRAIN = 32,
  BAR_COUNT = 33
};

struct Args {
  const float *A, *D, *dt_bias;
  const void* dt;
  long long dt0, dt1, dt2;
  const int* lengths;
  const float* init;           // states before the segments (slot stride) or, with one segment, before the first token; null: zero
  float* local;                // state kernel: slots of the own states
  float* decay;
  __nv_bfloat16* out;
  long long o0, o1, o2;
  int* device_status;
  int B, H, T, per;            // per: heads of a group
  int segments, seg_tokens, slots;
  bool softplus;
  int qg, qb, kg, kb, vh, vb;  // 0 where an axis is broadcast, else 1 (coordinates of the tensor maps)
};

__device__ __forceinline__ void tma_load_4d(void* dst, const void* tmap, uint64_t* bar, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(smem_u32(dst)), "l"(tmap), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_store_4d(const void* tmap, const void* src, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];\n\tcp.async.bulk.commit_group;"
               ::"l"(tmap), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
// 2^x to 2^-22 (what is below 2^-126 is zero)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 f2(uint32_t lo, uint32_t hi) { return make_float2(__uint_as_float(lo), __uint_as_float(hi)); }
__device__ __forceinline__ float2 unpack(uint32_t x) { return f2(x << 16, x & 0xffff0000u); }

// The wait of a whole warp: all lanes, or none.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort_flag));
}

struct Where {
  int b, h, g, bh, seg, t0, t1, live, tiles;
};
__device__ __forceinline__ Where where(const Args& a) {
  Where w;
  w.bh = blockIdx.x / a.segments;
  w.seg = blockIdx.x - w.bh * a.segments;
  w.b = w.bh / a.H;
  w.h = w.bh - w.b * a.H;
  w.g = w.h / a.per;
  w.t0 = w.seg * a.seg_tokens;
  w.t1 = min(w.t0 + a.seg_tokens, a.T);
  w.live = min(w.t1, sequence_length(a.lengths, w.b, a.T));
  w.tiles = w.live > w.t0 ? (w.live - w.t0 + CT - 1) / CT : 0;
  return w;
}

// Decays of every STRIDE-th tile from `first` on, one warp: a lane has four neighbouring tokens, eight lanes a block; the next tile's
// steps are on their way.  ALL: the factors of the weights too.  Returns the logarithm (base 2) of the decay over these tiles.
template <bool ALL, int STRIDE>
__device__ __forceinline__ double decay_warp(int first, const Args& a, const Where& w, Decays* slots, uint64_t* bars, volatile int* abort_flag, bool& ok) {
  const int lane = threadIdx.x & 31;
  const __nv_bfloat16* dt = static_cast<const __nv_bfloat16*>(a.dt) + w.b * a.dt0 + w.h * a.dt1;
  const float rate = (float)((double)a.A[w.h] * 1.4426950408889634074);
  const float bias = a.dt_bias != nullptr ? a.dt_bias[w.h] : 0.f;
  double all = 0.0;
  __nv_bfloat16 next[4];                         // (as they come: nothing waits for them before the next tile)
  auto fetch = [&](int j) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = w.t0 + j * CT + lane * 4 + i;
      next[i] = dt[(long long)min(t, w.live - 1) * a.dt2];
    }
  };
  if (first < w.tiles) fetch(first);
#pragma unroll 1
  for (int j = first; j < w.tiles; j += STRIDE) {
    float s[4], c[4], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = __bfloat162float(next[i]) + bias;
      s[i] = a.softplus ? softplus(x) : x;
      if (w.t0 + j * CT + lane * 4 + i >= w.live) s[i] = 0.f;
      sum = fmaf(s[i], rate, sum);
      c[i] = sum;
    }
    if (j + STRIDE < w.tiles) fetch(j + STRIDE);
    float upto = sum;                            // from the start of the block
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) {
      const float o = __shfl_up_sync(0xffffffffu, upto, off, 8);
      if ((lane & 7) >= off) upto += o;
    }
    // before this lane's tokens (their own sum taken off `upto` again would leave its rounding, 2^-3 where they lose 2^21); of the whole block
    float base = __shfl_up_sync(0xffffffffu, upto, 1, 8);
    if ((lane & 7) == 0) base = 0.f;
    const float mine = __shfl_sync(0xffffffffu, upto, 7, 8);
    // What a token loses up to the end of its block, summed from the end: as a difference it would carry the rounding of the whole
    // block's sum, 2^-19 of the weight where the block decays by 2^-50.
    float after = 0.f, lost[4];
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      lost[i] = after;
      after = fmaf(s[i], rate, after);
    }
    float from = after;
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) {
      const float o = __shfl_down_sync(0xffffffffu, from, off, 8);
      if ((lane & 7) + off < 8) from += o;
    }
    from = __shfl_down_sync(0xffffffffu, from, 1, 8);
    if ((lane & 7) == 7) from = 0.f;
    const float b0 = __shfl_sync(0xffffffffu, mine, 0), b1 = __shfl_sync(0xffffffffu, mine, 8), b2 = __shfl_sync(0xffffffffu, mine, 16),
                b3 = __shfl_sync(0xffffffffu, mine, 24);
    all += (double)b0 + b1 + b2 + b3;
    const int blk = lane >> 3, slot = j & (NSLOT - 1);
    const float behind = ex2(blk == 0 ? b1 + b2 + b3 : blk == 1 ? b2 + b3 : blk == 2 ? b3 : 0.f);
    ok = warp_wait(bars + BAR_DEC_EMPTY + slot, ((j / NSLOT) & 1) ^ 1, abort_flag);
    if (!ok) break;
    Decays& d = slots[slot];
    float tail[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[i] += base;
      tail[i] = s[i] * ex2(from + lost[i]);
    }
    reinterpret_cast<float4*>(d.left)[lane] = make_float4(tail[0] * behind, tail[1] * behind, tail[2] * behind, tail[3] * behind);
    if (ALL) {
      const float m = 0.5f * mine;
      reinterpret_cast<float4*>(d.tail)[lane] = make_float4(tail[0], tail[1], tail[2], tail[3]);
      reinterpret_cast<float4*>(d.row)[lane] = make_float4(ex2(c[0]), ex2(c[1]), ex2(c[2]), ex2(c[3]));
      reinterpret_cast<float4*>(d.inv)[lane] = make_float4(s[0] * ex2(m - c[0]), s[1] * ex2(m - c[1]), s[2] * ex2(m - c[2]), s[3] * ex2(m - c[3]));
      reinterpret_cast<float4*>(d.rel)[lane] = make_float4(c[0], c[1], c[2], c[3]);
      reinterpret_cast<float4*>(d.step)[lane] = make_float4(s[0], s[1], s[2], s[3]);
      if ((lane & 7) == 0) d.half[blk] = m;
      // lanes 0-3: before; 4: the whole tile; 5: [2][0], 6: [3][0], 7: [3][1]; neighbours are 1
      const float e = ex2(lane == 1 ? b0 : lane == 2 ? b0 + b1 : lane == 3 ? b0 + b1 + b2 : lane == 4 ? (b0 + b1) + (b2 + b3) : lane == 5 ? b1
                          : lane == 6 ? b1 + b2 : lane == 7 ? b2 : 0.f);
      if (lane < 4) d.before[lane] = e;
      if (lane == 4) d.total = e;
      if (lane >= 5 && lane < 8) d.between[lane == 5 ? 2 : 3][lane == 7 ? 1 : 0] = e;
      if (lane >= 8 && lane < 11) d.between[lane - 7][lane - 8] = 1.f;
    } else if (lane == 0) {
      d.total = ex2((b0 + b1) + (b2 + b3));
    }
    mbar_arrive(bars + BAR_DEC_FULL + slot);
  }
  return all;
}

// 8 bf16 entries times a weight: bf16 terms of the products, the first rounded, the next what it left.
template <int TERMS>
__device__ __forceinline__ void scaled_terms(const uint4& x, float w, uint4 (&out)[TERMS]) {
  const uint32_t in[4] = {x.x, x.y, x.z, x.w};
  uint32_t o[TERMS][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 p = mul_pair(unpack(in[i]), make_float2(w, w));
#pragma unroll
    for (int m = 0; m < TERMS; ++m) {
      o[m][i] = pack_bf16(p.x, p.y);
      if (m + 1 < TERMS) p = fma_pair(unpack(o[m][i]), make_float2(-1.f, -1.f), p);
    }
  }
#pragma unroll
  for (int m = 0; m < TERMS; ++m) out[m] = make_uint4(o[m][0], o[m][1], o[m][2], o[m][3]);
}

// Common start: barriers, TMEM.  Returns the aligned base of shared memory.
__device__ __forceinline__ unsigned char* aligned_base(unsigned char* raw) {
  return reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
}

// Row of the state that a thread of the state warps holds: n = 128 all lanes, n = 64 the first 16 lanes of each warp (the lanes that a
// product of 64 rows has).
template <int N> __device__ __forceinline__ int state_row(int q4, int lane) { return N == 128 ? q4 * 32 + lane : q4 * 16 + lane; }
template <int N> __device__ __forceinline__ bool state_lane(int lane) { return N == 128 || lane < 16; }

template <int N>
__global__ void __launch_bounds__(kOutThreads, 1)
tc_ssm_out_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ CUtensorMap tmO, const __grid_constant__ Args a) {
  typedef Shape<N, 0> Sh;
  constexpr int NST = Sh::NST, XB = Sh::XB, KS = N / 16;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = aligned_base(smem_raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + Sh::OFF_BAR);
  Decays* decays = reinterpret_cast<Decays*>(base + Sh::OFF_DEC);
  auto qtile = [&](int s) { return base + s * Sh::STAGE; };
  auto ktile = [&](int s) { return base + s * Sh::STAGE + Sh::K_OFF; };
  auto vtile = [&](int s) { return base + s * Sh::STAGE + Sh::V_OFF; };
  auto xtile = [&](int j) { return base + Sh::OFF_X + (XB == 2 ? (j & 1) : 0) * HALF; };
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  bool ok = true;

  if (tid == 0) {
    abort_s = 0;
    for (int i = 0; i < BAR_COUNT; ++i) {
      uint32_t n = 1;
      if (i >= BAR_EMPTY && i < BAR_EMPTY + 3) n = 2 + 8;
      if (i >= BAR_DEC_FULL && i < BAR_DEC_FULL + NSLOT) n = 32;
      if (i >= BAR_DEC_EMPTY && i < BAR_DEC_EMPTY + NSLOT) n = 4 + 8 + 8;
      if (i == BAR_P_FULL || i == BAR_P_FULL + 1 || i == BAR_O_EMPTY || i == BAR_X_FULL || i == BAR_X_FULL + 1) n = 256;
      if (i == BAR_SL_EMPTY || i == BAR_ST) n = 128;
      if (i == BAR_O_FULL || i == BAR_DRAIN) n = 2;
      mbar_init(bars + i, n);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
    tma_prefetch_desc(&tmO);
  }
  if (warp == 0) {
    tmem_alloc(&tmem_base_s, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = tmem_base_s;
  wait_for_kernels_ahead();
  const Where w = where(a);

  if (warp == 0) {
    // =========================== decays ===========================
    decay_warp<true, 1>(0, a, w, decays, bars, abort_flag, ok);
  } else if (warp == 1) {
    // =========================== scores Q K^T, one tile ahead, and Q S ===========================
    const uint32_t id_qk = instr_desc(kFmtBF16, kFmtBF16, 0, 0, 128, 128), id_r = instr_desc(kFmtBF16, kFmtBF16, 0, 1, 128, DV);
    const uint64_t dk = smem_desc(0, 16, 1024, kSwizzle128B), dn = smem_desc(0, HALF, 1024, kSwizzle128B);
    const uint32_t st = smem_u32(base + Sh::OFF_S);
    int s = 0, s_before = 0, round = 0;
#pragma unroll 1
    for (int j = 0; j <= w.tiles && ok; ++j) {
      if (j < w.tiles) {
        const int b = j & 1;
        ok = warp_wait(bars + BAR_FULL + s, round & 1, abort_flag) && warp_wait(bars + BAR_P_EMPTY + b, ((j >> 1) & 1) ^ 1, abort_flag);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t qa = smem_u32(qtile(s)), ka = smem_u32(ktile(s));
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < KS; ++ks)
            mma_f16_ss(tb + COL_P + b * 128, at(dk, qa + (ks >> 2) * HALF + (ks & 3) * 32), at(dk, ka + (ks >> 2) * HALF + (ks & 3) * 32), id_qk, ks > 0);
          mma_commit(bars + BAR_S_FULL + b);
        }
        __syncwarp();
      }
      if (j > 0) {
        // the state before the tile is in place, the result of the tile before it has been read
        ok = warp_wait(bars + BAR_ST, (j - 1) & 1, abort_flag) && warp_wait(bars + BAR_O_EMPTY, j & 1, abort_flag);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t qa = smem_u32(qtile(s_before));
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < KS; ++ks)
            mma_f16_ss(tb + COL_R, at(dk, qa + (ks >> 2) * HALF + (ks & 3) * 32), at(dn, st + ks * 2048), id_r, ks > 0);
          mma_commit(bars + BAR_R_DONE);
          mma_commit(bars + BAR_O_FULL);
          mma_commit(bars + BAR_EMPTY + s_before);
        }
        __syncwarp();
      }
      s_before = s;
      if (++s == NST) {
        s = 0;
        ++round;
      }
    }
  } else if (warp == 2) {
    // =========================== own state of the tile K^T V', product with V ===========================
    const uint32_t id_s = instr_desc(kFmtBF16, kFmtBF16, 1, 1, N, DV), id_v = instr_desc(kFmtBF16, kFmtBF16, 0, 1, 128, DV);
    const uint64_t dn = smem_desc(0, HALF, 1024, kSwizzle128B);
    int s = 0, round = 0;
#pragma unroll 1
    for (int j = 0; j < w.tiles && ok; ++j) {
      const int b = j & 1;
      ok = warp_wait(bars + BAR_FULL + s, round & 1, abort_flag) &&
           warp_wait(bars + BAR_X_FULL + (XB == 2 ? b : 0), (XB == 2 ? j >> 1 : j) & 1, abort_flag);
      if (ok && j + 1 < w.tiles) {
        ok = warp_wait(bars + BAR_SL_EMPTY, (j & 1) ^ 1, abort_flag);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t ka = smem_u32(ktile(s)), xa = smem_u32(xtile(j));
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < CT / 16; ++ks) mma_f16_ss(tb + COL_SL, at(dn, ka + ks * 2048), at(dn, xa + ks * 2048), id_s, ks > 0);
          mma_commit(bars + BAR_SL_FULL);
          mma_commit(bars + BAR_X_EMPTY + (XB == 2 ? b : 0));
        }
        __syncwarp();
      }
      ok = ok && warp_wait(bars + BAR_P_FULL + b, (j >> 1) & 1, abort_flag) && warp_wait(bars + BAR_O_EMPTY, (j & 1) ^ 1, abort_flag);
      if (!ok) break;
      if (elect_one()) {
        const uint32_t va = smem_u32(vtile(s));
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < CT / 16; ++ks)
          mma_f16_ts(tb + COL_Y, tb + COL_P + b * 128 + (ks >> 2) * 64 + (ks & 3) * 8, at(dn, va + ks * 2048), id_v, ks > 0);
        mma_commit(bars + BAR_P_EMPTY + b);
        mma_commit(bars + BAR_O_FULL);
        mma_commit(bars + BAR_EMPTY + s);
      }
      __syncwarp();
      if (++s == NST) {
        s = 0;
        ++round;
      }
    }
  } else if (warp == 3) {
    // =========================== TMA loads ===========================
    if (lane == 0) {
      int asked = 0;
      for (int j = 0; j < w.tiles && ok; ++j) {
        const int s = j % NST, tok = w.t0 + j * CT;
        ok = wait_or_abort(bars + BAR_EMPTY + s, ((j / NST) & 1) ^ 1, abort_flag);
        if (!ok) break;
        ++asked;
        mbar_arrive_expect_tx(bars + BAR_FULL + s, Sh::STAGE);
#pragma unroll
        for (int i = 0; i < Sh::HALVES; ++i) {
          tma_load_4d(qtile(s) + i * HALF, &tmQ, bars + BAR_FULL + s, i * 64, tok, w.g * a.qg, w.b * a.qb);
          tma_load_4d(ktile(s) + i * HALF, &tmK, bars + BAR_FULL + s, i * 64, tok, w.g * a.kg, w.b * a.kb);
        }
        tma_load_4d(vtile(s), &tmV, bars + BAR_FULL + s, 0, tok, w.h * a.vh, w.b * a.vb);
      }
      for (int j = max(0, asked - NST); j < asked; ++j) mbar_wait(bars + BAR_FULL + j % NST, (j / NST) & 1);     // none is in flight when the CTA ends
    }
  } else if (warp < W_WEIGHT0) {
    // =========================== state ===========================
    // fp32 in TMEM (in registers it would take 64 of a thread's 80)
    const int q4 = warp & 3, row = state_row<N>(q4, lane);
    const bool mine = state_lane<N>(lane);
    const uint32_t scol = tmem_addr(tb, q4 * 32, COL_S), lcol = tmem_addr(tb, q4 * 32, COL_SL);
    const float* src = a.init != nullptr ? a.init + ((size_t)w.bh * a.slots + w.seg) * (N * DV) + (size_t)row * DV : nullptr;
    // j: the tile that the state goes before (0: as handed in; then the own state of tile j - 1 is added)
#pragma unroll 1
    for (int j = 0; j < w.tiles && ok; ++j) {
      float total = 0.f;
      if (j > 0) {
        const int slot = (j - 1) & (NSLOT - 1);
        ok = warp_wait(bars + BAR_DEC_FULL + slot, ((j - 1) / NSLOT) & 1, abort_flag);
        if (!ok) break;
        total = decays[slot].total;
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + BAR_DEC_EMPTY + slot);
        ok = warp_wait(bars + BAR_SL_FULL, (j - 1) & 1, abort_flag) && warp_wait(bars + BAR_R_DONE, (j - 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
      }
      const float2 keep = make_float2(total, total);
#pragma unroll 1
      for (int p = 0; p < 4; ++p) {
        uint32_t S[16];
        if (j > 0) {
          uint32_t x[16];
          tmem_ld16(scol + p * 16, S);
          tmem_ld16(lcol + p * 16, x);
          tmem_wait_ld(S);
          tmem_wait_ld(x);
#pragma unroll
          for (int c = 0; c < 16; c += 2) {
            const float2 n = fma_pair(keep, f2(S[c], S[c + 1]), f2(x[c], x[c + 1]));
            S[c] = __float_as_uint(n.x);
            S[c + 1] = __float_as_uint(n.y);
          }
        } else {
#pragma unroll
          for (int c = 0; c < 16; c += 4) {
            const float4 x = mine && src != nullptr ? *reinterpret_cast<const float4*>(src + p * 16 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
            S[c] = __float_as_uint(x.x);
            S[c + 1] = __float_as_uint(x.y);
            S[c + 2] = __float_as_uint(x.z);
            S[c + 3] = __float_as_uint(x.w);
          }
        }
        tmem_st16(scol + p * 16, S);
        if (mine) {                              // the bf16 copy that the Q S of tile j reads: [row][64 columns]
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pack_bf16(__uint_as_float(S[8 * c + 2 * i]), __uint_as_float(S[8 * c + 2 * i + 1]));
            *reinterpret_cast<uint4*>(base + Sh::OFF_S + sw128_offset(row, 2 * p + c)) = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
      }
      tmem_wait_st();
      tc_fence_before();
      if (j > 0) mbar_arrive(bars + BAR_SL_EMPTY);
      fence_async_smem();
      mbar_arrive(bars + BAR_ST);
    }
  } else if (warp < W_OUT0) {
    // =========================== weights (256 threads) ===========================
    const uint32_t q4 = warp & 3;
    const int ch = (warp - W_WEIGHT0) >> 2;      // column half
    const int row = q4 * 32 + lane;              // token of the tile (= TMEM lane)
#pragma unroll 1
    for (int j = 0; j < w.tiles && ok; ++j) {
      const int b = j & 1, slot = j & (NSLOT - 1);
      ok = warp_wait(bars + BAR_DEC_FULL + slot, (j / NSLOT) & 1, abort_flag) && warp_wait(bars + BAR_S_FULL + b, (j >> 1) & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const Decays& d = decays[slot];
      const float rf = d.row[row], rel = d.rel[row];
      const uint32_t scol = tmem_addr(tb, q4 * 32, COL_P + b * 128 + ch * 64);
      // Blocks of 32 columns; the bf16 weights go over the scores of this thread's half, which have been read by then.
#pragma unroll 1
      for (int hf = 0; hf < 2; ++hf) {
        const uint32_t blk = 2 * ch + hf;
        uint32_t pk[16];
        if (blk > q4) {
#pragma unroll
          for (int c = 0; c < 16; ++c) pk[c] = 0u;
        } else {
          uint32_t y[32];
          tmem_ld32(scol + hf * 32, y);
          const bool diag = blk == q4;
          const float4* col = reinterpret_cast<const float4*>((diag ? d.inv : d.tail) + blk * 32);
          const float f = diag ? ex2(rel - d.half[blk]) : rf * d.between[q4][blk];
          const float2 ff = make_float2(f, f);
          // A block is steep where a factor leaves fp32's normal range, the step size with it: 1000 2^119 would be inf, 2^-20 2^-118
          // has lost bits or is zero, and so would be their product with the row's factor, which is s_i itself on the diagonal.
          // Every lane looks at its own token.  (Here and not where the factors are formed: that warp's instructions count, and the
          // test there took 8 x 16 heads x 4096 tokens from 59.3 us to 62.9.)
          bool steep = false;
          if (diag) {
            const float inv = fabsf(d.inv[row]);
            steep = __any_sync(0xffffffffu, !(fabsf(rel - d.half[blk]) < 120.f && (d.step[row] == 0.f || (inv >= 0x1p-126f && inv < 0x1p126f))));
          }
          tmem_wait_ld(y);
          if (steep) {
            // Column by column from the diagonal backwards, what a token loses to the row summed on the way: as a difference of sums
            // from the block's start it would carry the rounding of a token that forgets everything (18 % where that loses 2^21).
            const float rate = a.A[w.h] * 1.44269504f;
            float lost = 0.f;
#pragma unroll
            for (int c = 30; c >= 0; c -= 2) {
              const float s1 = d.step[blk * 32 + c + 1], s0 = d.step[blk * 32 + c], w1 = s1 * ex2(lost);
              if (c + 1 <= lane) lost = fmaf(s1, rate, lost);
              const float w0 = s0 * ex2(lost);
              if (c <= lane) lost = fmaf(s0, rate, lost);
              pk[c / 2] = pack_bf16(__uint_as_float(y[c]) * w0, __uint_as_float(y[c + 1]) * w1);
            }
          } else {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              const float4 cf = col[c / 4];
              const float2 u = mul_pair(mul_pair(make_float2(cf.x, cf.y), ff), f2(y[c], y[c + 1])), v = mul_pair(mul_pair(make_float2(cf.z, cf.w), ff), f2(y[c + 2], y[c + 3]));
              pk[c / 2] = pack_bf16(u.x, u.y);
              pk[c / 2 + 1] = pack_bf16(v.x, v.y);
            }
          }
          if (diag) {                            // column c counts for rows c and behind
#pragma unroll
            for (int c = 0; c < 16; ++c) pk[c] = 2 * c + 1 <= lane ? pk[c] : 2 * c == lane ? pk[c] & 0xffffu : 0u;
          }
        }
        tmem_st16(scol + hf * 16, pk);
      }
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(bars + BAR_P_FULL + b);
      if (lane == 0) mbar_arrive(bars + BAR_DEC_EMPTY + slot);
    }
  } else {
    // =========================== scaled V, epilogue (256 threads) ===========================
    const uint32_t q4 = warp & 3;
    const int ch = (warp - W_OUT0) >> 2;         // column half
    const int row = q4 * 32 + lane;              // token of the tile (= TMEM lane)
    const float skip = a.D != nullptr ? a.D[w.h] : 0.f;
    unsigned char* rows = base + Sh::OFF_OUT + (warp - W_OUT0) * 2048;
    float from_state = 0.f;                      // 2^(c_t) from the start of the tile
    int s = 0, s_before = 0, round = 0;
#pragma unroll 1
    for (int j = 0; j <= w.tiles && ok; ++j) {
      float from_here = 0.f;
      if (j < w.tiles) {
        const int b = j & 1, slot = j & (NSLOT - 1), xb = XB == 2 ? b : 0;
        ok = warp_wait(bars + BAR_FULL + s, round & 1, abort_flag) && warp_wait(bars + BAR_DEC_FULL + slot, (j / NSLOT) & 1, abort_flag) &&
             warp_wait(bars + BAR_X_EMPTY + xb, ((XB == 2 ? j >> 1 : j) & 1) ^ 1, abort_flag);
        if (!ok) break;
        const float left = decays[slot].left[row];
        from_here = decays[slot].row[row] * decays[slot].before[q4];
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + BAR_DEC_EMPTY + slot);
        const bool dead = w.t0 + j * CT + row >= w.live;
#pragma unroll 2
        for (int c = 4 * ch; c < 4 * ch + 4; ++c) {
          const uint32_t off = sw128_offset(row, c);
          uint4 x[1], v = *reinterpret_cast<const uint4*>(vtile(s) + off);
          if (dead) {                            // what lies behind the sequence's end becomes zero
            v = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(vtile(s) + off) = v;
#pragma unroll
            for (int i = 0; i < Sh::HALVES; ++i) *reinterpret_cast<uint4*>(ktile(s) + i * HALF + off) = v;
          }
          scaled_terms<1>(v, left, x);
          *reinterpret_cast<uint4*>(xtile(j) + off) = x[0];
        }
        fence_async_smem();
        mbar_arrive(bars + BAR_X_FULL + xb);
      }
      if (j > 0) {
        ok = warp_wait(bars + BAR_O_FULL, (j - 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (lane == 0) bulk_wait_read();         // the store of the tile before has read the staging rows
        __syncwarp();
        const bool dead = w.t0 + (j - 1) * CT + row >= w.live;
        const float2 f = make_float2(from_state, from_state), sk = make_float2(skip, skip);
#pragma unroll 1
        for (int p = 0; p < 2; ++p) {
          uint32_t y[16], r[16];
          tmem_ld16(tmem_addr(tb, q4 * 32, COL_Y + ch * 32 + p * 16), y);
          tmem_ld16(tmem_addr(tb, q4 * 32, COL_R + ch * 32 + p * 16), r);
          const unsigned char* vrow = vtile(s_before);
          const uint4 v0 = *reinterpret_cast<const uint4*>(vrow + sw128_offset(row, 4 * ch + 2 * p));
          const uint4 v1 = *reinterpret_cast<const uint4*>(vrow + sw128_offset(row, 4 * ch + 2 * p + 1));
          const uint32_t in[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
          tmem_wait_ld(y);
          tmem_wait_ld(r);
          uint32_t o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 z = fma_pair(unpack(in[i]), sk, fma_pair(f, f2(r[2 * i], r[2 * i + 1]), f2(y[2 * i], y[2 * i + 1])));
            o[i] = dead ? 0u : pack_bf16(z.x, z.y);
          }
          *reinterpret_cast<uint4*>(rows + lane * 64 + (((2 * p) ^ ((lane >> 1) & 3)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
          *reinterpret_cast<uint4*>(rows + lane * 64 + (((2 * p + 1) ^ ((lane >> 1) & 3)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
        }
        tc_fence_before();
        mbar_arrive(bars + BAR_O_EMPTY);
        fence_async_smem();
        __syncwarp();
        const int first = w.t0 + (j - 1) * CT + (int)q4 * 32;
        if (lane == 0) {
          mbar_arrive(bars + BAR_EMPTY + s_before);
          if (first < a.T) tma_store_4d(&tmO, rows, ch * 32, first, w.h, w.b);
        }
      }
      from_state = from_here;
      s_before = s;
      if (++s == NST) {
        s = 0;
        ++round;
      }
    }
  }

  // ---------------- teardown ----------------
  if (!ok && a.device_status != nullptr) atomicExch(a.device_status, (int)KATA_ERR_DEVICE_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if ((warp == 1 || warp == 2) && elect_one()) {
    mma_commit(bars + BAR_DRAIN);
    mbar_wait(bars + BAR_DRAIN, 0);
  }
  if (warp >= W_OUT0 && lane == 0) bulk_wait();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tb, TMEM_COLS);
  // rows behind the last tile of the sequence
  const int first = w.t0 + w.tiles * CT;
  for (long long i = tid; i < (long long)(w.t1 - first) * 8; i += kOutThreads)
    *reinterpret_cast<uint4*>(a.out + w.b * a.o0 + w.h * a.o1 + (first + (i >> 3)) * a.o2 + (i & 7) * 8) = make_uint4(0u, 0u, 0u, 0u);
}

template <int N, int TERMS>
__global__ void __launch_bounds__(kStateThreads, 1)
tc_ssm_state_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Args a) {
  typedef Shape<N, TERMS> Sh;
  constexpr int NST = Sh::NST;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = aligned_base(smem_raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + Sh::OFF_BAR);
  Decays* decays = reinterpret_cast<Decays*>(base + Sh::OFF_DEC);
  auto ktile = [&](int s) { return base + s * Sh::STAGE; };
  auto vtile = [&](int s) { return base + s * Sh::STAGE + Sh::V_OFF; };
  auto xtile = [&](int j, int term) { return base + Sh::OFF_X + ((j & 1) * TERMS + term) * HALF; };
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  __shared__ double all_s[2];                    // logarithms of the decay over the two warps' tiles
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  bool ok = true;
  if ((int)(blockIdx.x % (unsigned)a.segments) + 2 > a.slots) return;      // (the last segment's own state is not wanted)

  if (tid == 0) {
    abort_s = 0;
    for (int i = 0; i < BAR_COUNT; ++i) {
      uint32_t n = 1;
      if (i >= BAR_DEC_FULL && i < BAR_DEC_FULL + NSLOT) n = 32;
      if (i >= BAR_DEC_EMPTY && i < BAR_DEC_EMPTY + NSLOT) n = 12;
      if (i == BAR_X_FULL || i == BAR_X_FULL + 1) n = 256;
      if (i == BAR_SL_EMPTY || i == BAR_SL_EMPTY + 1) n = 128;
      mbar_init(bars + i, n);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 0) {
    tmem_alloc(&tmem_base_s, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = tmem_base_s;
  wait_for_kernels_ahead();
  const Where w = where(a);

  if (warp == 0) {
    // =========================== TMA loads ===========================
    if (lane == 0) {
      int asked = 0;
      for (int j = 0; j < w.tiles && ok; ++j) {
        const int s = j % NST, tok = w.t0 + j * CT;
        ok = wait_or_abort(bars + BAR_EMPTY + s, ((j / NST) & 1) ^ 1, abort_flag);
        if (!ok) break;
        ++asked;
        mbar_arrive_expect_tx(bars + BAR_FULL + s, Sh::STAGE);
#pragma unroll
        for (int i = 0; i < Sh::HALVES; ++i) tma_load_4d(ktile(s) + i * HALF, &tmK, bars + BAR_FULL + s, i * 64, tok, w.g * a.kg, w.b * a.kb);
        tma_load_4d(vtile(s), &tmV, bars + BAR_FULL + s, 0, tok, w.h * a.vh, w.b * a.vb);
      }
      for (int j = max(0, asked - NST); j < asked; ++j) mbar_wait(bars + BAR_FULL + j % NST, (j / NST) & 1);     // none is in flight when the CTA ends
    }
  } else if (warp == 1) {
    // =========================== own state of the tile K^T V' ===========================
    const uint32_t id_s = instr_desc(kFmtBF16, kFmtBF16, 1, 1, N, DV);
    const uint64_t dn = smem_desc(0, HALF, 1024, kSwizzle128B);
    for (int j = 0; j < w.tiles && ok; ++j) {
      const int s = j % NST, b = j & 1;
      ok = warp_wait(bars + BAR_FULL + s, (j / NST) & 1, abort_flag) && warp_wait(bars + BAR_X_FULL + b, (j >> 1) & 1, abort_flag) &&
           warp_wait(bars + BAR_SL_EMPTY + b, ((j >> 1) & 1) ^ 1, abort_flag);
      if (!ok) break;
      if (elect_one()) {
        const uint32_t ka = smem_u32(ktile(s));
        tc_fence_after();
#pragma unroll
        for (int m = TERMS - 1; m >= 0; --m) {           // (the small terms first)
          const uint32_t xa = smem_u32(xtile(j, m));
#pragma unroll
          for (int ks = 0; ks < CT / 16; ++ks)
            mma_f16_ss(tb + COL_SL + b * DV, at(dn, ka + ks * 2048), at(dn, xa + ks * 2048), id_s, m + 1 < TERMS || ks > 0);
        }
        mma_commit(bars + BAR_SL_FULL + b);
        mma_commit(bars + BAR_X_EMPTY + b);
        mma_commit(bars + BAR_EMPTY + s);
      }
      __syncwarp();
    }
  } else if (warp < W_STATE0) {
    // =========================== decays, every other tile ===========================
    const double part = decay_warp<false, 2>(warp - 2, a, w, decays, bars, abort_flag, ok);
    if (lane == 0) all_s[warp - 2] = part;
  } else if (warp >= W_STATE0 && warp < W_WEIGHT0) {
    // =========================== state ===========================
    const int q4 = warp & 3, row = state_row<N>(q4, lane);
    float2 S[DV / 2];
#pragma unroll
    for (int c = 0; c < DV / 2; ++c) S[c] = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int j = 0; j < w.tiles && ok; ++j) {
      const int b = j & 1, slot = j & (NSLOT - 1);
      ok = warp_wait(bars + BAR_DEC_FULL + slot, (j / NSLOT) & 1, abort_flag);
      const float total = ok ? decays[slot].total : 0.f;
      __syncwarp();
      if (lane == 0) mbar_arrive(bars + BAR_DEC_EMPTY + slot);
      ok = ok && warp_wait(bars + BAR_SL_FULL + b, (j >> 1) & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint32_t x[32];
        tmem_ld32(tmem_addr(tb, q4 * 32, COL_SL + b * DV + hf * 32), x);
        tmem_wait_ld(x);
#pragma unroll
        for (int c = 0; c < 16; ++c) S[hf * 16 + c] = fma_pair(make_float2(total, total), S[hf * 16 + c], f2(x[2 * c], x[2 * c + 1]));
      }
      tc_fence_before();
      mbar_arrive(bars + BAR_SL_EMPTY + b);
    }
    if (state_lane<N>(lane)) {
      float4* dst = reinterpret_cast<float4*>(a.local + ((size_t)w.bh * a.slots + w.seg + 1) * (N * DV) + (size_t)row * DV);
#pragma unroll
      for (int c = 0; c < DV / 4; ++c) dst[c] = make_float4(S[2 * c].x, S[2 * c].y, S[2 * c + 1].x, S[2 * c + 1].y);
    }
  } else if (warp >= W_WEIGHT0) {
    // =========================== scaled V in three terms ===========================
    const int q4 = warp & 3, ch = (warp - W_WEIGHT0) >> 2, tok = q4 * 32 + lane;
    for (int j = 0; j < w.tiles && ok; ++j) {
      const int s = j % NST, b = j & 1, slot = j & (NSLOT - 1);
      ok = warp_wait(bars + BAR_DEC_FULL + slot, (j / NSLOT) & 1, abort_flag);
      const float left = ok ? decays[slot].left[tok] : 0.f;
      __syncwarp();
      if (lane == 0) mbar_arrive(bars + BAR_DEC_EMPTY + slot);
      ok = ok && warp_wait(bars + BAR_FULL + s, (j / NST) & 1, abort_flag) && warp_wait(bars + BAR_X_EMPTY + b, ((j >> 1) & 1) ^ 1, abort_flag);
      if (!ok) break;
      const bool dead = w.t0 + j * CT + tok >= w.live;
#pragma unroll
      for (int c = 4 * ch; c < 4 * ch + 4; ++c) {
        const uint32_t off = sw128_offset(tok, c);
        uint4 v = *reinterpret_cast<const uint4*>(vtile(s) + off), x[TERMS];
        if (dead) {                              // (K times zero has to be zero, whatever lies there)
          v = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int i = 0; i < Sh::HALVES; ++i) *reinterpret_cast<uint4*>(ktile(s) + i * HALF + off) = v;
        }
        scaled_terms<TERMS>(v, left, x);
#pragma unroll
        for (int m = 0; m < TERMS; ++m) *reinterpret_cast<uint4*>(xtile(j, m) + off) = x[m];
      }
      fence_async_smem();
      mbar_arrive(bars + BAR_X_FULL + b);
    }
  }

  // ---------------- teardown ----------------
  if (!ok && a.device_status != nullptr) atomicExch(a.device_status, (int)KATA_ERR_DEVICE_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1 && elect_one()) {
    mma_commit(bars + BAR_DRAIN);
    mbar_wait(bars + BAR_DRAIN, 0);
  }
  __syncthreads();
  if (warp == 0) tmem_dealloc(tb, TMEM_COLS);
  if (tid == 0) a.decay[(size_t)w.bh * a.slots + w.seg] = ex2((float)(all_s[0] + all_s[1]));
}

// [B][heads][T][width] bf16 view, box = cols x rows x 1 x 1; axes that are broadcast (stride 0) have one entry and a coordinate of 0.
bool make_view_map(CUtensorMap* tm, const View& v, int B, int heads, int T, int width, int cols, int rows, int* head_on, int* batch_on) {
  EncodeTiledFn fn = tensor_map_encoder();
  if (fn == nullptr) return false;
  *head_on = v.s1 != 0;
  *batch_on = v.s0 != 0;
  const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)T, (cuuint64_t)(v.s1 != 0 ? heads : 1), (cuuint64_t)(v.s0 != 0 ? B : 1)};
  const cuuint64_t strides[3] = {(cuuint64_t)(T > 1 ? v.s2 * 2 : 16), (cuuint64_t)(v.s1 != 0 ? v.s1 * 2 : 16), (cuuint64_t)(v.s0 != 0 ? v.s0 * 2 : 16)};
  const cuuint32_t box[4] = {(cuuint32_t)cols, (cuuint32_t)rows, 1, 1}, es[4] = {1, 1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, v.p, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int N> void launch(const Ssm& a, const SsmPlan& plan, float* ws, int* device_status, LaunchCtx& ctx) {
  CUtensorMap tmQ, tmK, tmV, tmO;
  Args r = {};
  int on[2];
  if (!make_view_map(&tmQ, a.q, a.B, a.G, a.T, N, 64, CT, &r.qg, &r.qb) || !make_view_map(&tmK, a.k, a.B, a.G, a.T, N, 64, CT, &r.kg, &r.kb) ||
      !make_view_map(&tmV, a.v, a.B, a.H, a.T, DV, 64, CT, &r.vh, &r.vb) || !make_view_map(&tmO, a.out, a.B, a.H, a.T, DV, 32, 32, &on[0], &on[1]) ||
      !allow_smem<tc_ssm_out_kernel<N>>((int)Shape<N, 0>::SMEM) || !allow_smem<tc_ssm_state_kernel<N, 1>>((int)Shape<N, 1>::SMEM) ||
      !allow_smem<tc_ssm_state_kernel<N, 3>>((int)Shape<N, 3>::SMEM)) {
    ctx.status = KATA_ERR_CUDA;
    return;
  }
  r.A = a.A; r.D = a.D; r.dt_bias = a.dt_bias;
  r.dt = a.dt.p; r.dt0 = a.dt.s0; r.dt1 = a.dt.s1; r.dt2 = a.dt.s2;
  r.lengths = a.lengths;
  r.out = reinterpret_cast<__nv_bfloat16*>(a.out.p); r.o0 = a.out.s0; r.o1 = a.out.s1; r.o2 = a.out.s2;
  r.device_status = device_status;
  r.B = a.B; r.H = a.H; r.T = a.T; r.per = a.H / a.G;
  r.segments = plan.segments; r.seg_tokens = plan.seg_tokens;
  r.softplus = a.softplus;
  const dim3 grid((unsigned)(a.B * a.H) * plan.segments);
  const bool states = plan.segments > 1 || a.s_final != nullptr;
  r.slots = states ? plan.segments + (a.s_final != nullptr ? 1 : 0) : 1;
  r.init = a.s_init;
  if (states) {
    r.local = ws;
    r.decay = ws + (size_t)a.B * a.H * r.slots * (N * DV);
    // a final state: to the precision of fp32; states that only outputs read, through their bf16 copy: one term
    if (a.s_final != nullptr) launch_after(ctx, tc_ssm_state_kernel<N, 3>, grid, dim3(kStateThreads), Shape<N, 3>::SMEM, tmK, tmV, r);
    else launch_after(ctx, tc_ssm_state_kernel<N, 1>, grid, dim3(kStateThreads), Shape<N, 1>::SMEM, tmK, tmV, r);
    ssm_prefix(a, plan, r.slots, ws, ctx);
    r.init = ws;
  }
  launch_after(ctx, tc_ssm_out_kernel<N>, grid, dim3(kOutThreads), Shape<N, 0>::SMEM, tmQ, tmK, tmV, tmO, r);
}

}  // namespace

bool tc_ssm_supported(int dtype, int n, int d) { return dtype == KATA_BF16 && (n == 64 || n == 128) && d == DV; }

void tc_ssm(const Ssm& a, const SsmPlan& plan, float* ws, int* device_status, LaunchCtx& ctx) {
  if (a.n == 64) launch<64>(a, plan, ws, device_status, ctx);
  else launch<128>(a, plan, ws, device_status, ctx);
}

}  // namespace kata
