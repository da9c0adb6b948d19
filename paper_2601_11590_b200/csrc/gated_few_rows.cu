// The gated block for one token and a handful of tokens (bf16): bound by reading the weights once.
//
// A block owns 8 output columns of the gated product (8 gate rows and the 8 up rows of the same columns: one 16-row
// operand tile, so a thread ends up holding both projections of its columns), or 8 or 16 output columns of the projection
// behind it.  Its warps share the contraction: warp w takes every kWarps-th chunk of 32 steps, so that the block reads
// contiguous pieces of its weight rows, and the warps' sums are added in shared memory, always in the same order.
// Weights go from global memory straight into matrix fragments: the contraction may be taken in any order as long as both
// operands share it, so a thread loads 16 contiguous bytes of a weight row and of a token's row and uses them as the
// fragments of two products (mma.sync, tokens as the 8-wide side).  tcgen05 has nothing to add here: its products would
// have to be staged through shared memory, and the matrix pipe is idle most of the time either way.
// Token rows beyond the last and weight rows beyond the last are read from the last valid row; their results are not stored.
#include "gated.cuh"

namespace epd {
namespace {

constexpr int kWarps = 8;
constexpr int kChunk = 32;          // contraction steps of a warp's chunk: 64 bytes of a row

enum { KIND_GATED = 0, KIND_16 = 1, KIND_8 = 2 };

struct FewRows {
  const __nv_bfloat16 *x, *w, *bias;
  int64_t ldx, ldw;
  int M, N, K;
  __nv_bfloat16* out;               // GATED: [M, N]; else bf16 out, or NULL
  float* out_f32;                   // else float out, or NULL
  int64_t ldo;
  __nv_bfloat16* pre;               // GATED: [M, 2N] or NULL
  int64_t ldp;
  int gate;
  int accumulate;
  int weights_settled;              // the kernel in front of this one started after everything that may write the weights
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_stream(const __nv_bfloat16* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

template <int KIND, int NT>
__global__ void __launch_bounds__(32 * kWarps, NT >= 2 ? 2 : 3)
few_rows_kernel(const FewRows p) {
  constexpr int COLS = KIND == KIND_16 ? 16 : 8;       // output columns of a block
  constexpr int kAhead = NT >= 4 ? 2 : 4;              // chunks loaded ahead of their products
  __shared__ float part[kWarps][NT * 8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * COLS;
  const int64_t r0 = min(n0 + g, p.N - 1);
  const int64_t r1 = KIND == KIND_GATED ? p.N + r0 : min(n0 + g + 8, p.N - 1);
  const __nv_bfloat16* w0 = p.w + r0 * p.ldw + 8 * t;
  const __nv_bfloat16* w1 = p.w + r1 * p.ldw + 8 * t;
  const __nv_bfloat16* xr[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) xr[j] = p.x + (int64_t)min(8 * j + g, p.M - 1) * p.ldx + 8 * t;

  float acc[NT][4] = {};
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 a0[kAhead], a1[kAhead];
  auto load_weights = [&](int k, uint4& u, uint4& v) {
    const bool in = k + 8 * t < p.K;                   // K is a multiple of 8: a 16-byte piece is whole or beyond the end
    u = in ? load_stream(w0 + k) : zero;
    v = in && KIND != KIND_8 ? load_stream(w1 + k) : zero;
  };
  constexpr int kStride = kWarps * kChunk;
  int k = warp * kChunk;
  // Behind the block's own gated kernel the weights may be fetched before that kernel has finished.
  if (p.weights_settled) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_weights(k + i * kStride, a0[i], a1[i]);
    pdl_wait();
  } else {
    pdl_wait();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_weights(k + i * kStride, a0[i], a1[i]);
  }
  // From here on whatever ran in front of this kernel has completed: the next one may start and fetch its weights.
  pdl_launch_dependents();
  for (; k < p.K; k += kAhead * kStride) {
    uint4 b[kAhead][NT];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool in = k + i * kStride + 8 * t < p.K;
#pragma unroll
      for (int j = 0; j < NT; ++j) b[i][j] = in ? *reinterpret_cast<const uint4*>(xr[j] + k + i * kStride) : zero;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint4 u = a0[i], v = a1[i];
      load_weights(k + (kAhead + i) * kStride, a0[i], a1[i]);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        mma_16816(acc[j], u.x, v.x, u.y, v.y, b[i][j].x, b[i][j].y);
        mma_16816(acc[j], u.z, v.z, u.w, v.w, b[i][j].z, b[i][j].w);
      }
    }
  }
  // fragment: acc[j][0..1] = (weight row g, tokens 8j + 2t, + 1), acc[j][2..3] = (weight row g + 8, same tokens)
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[warp][8 * j + 2 * t + (e & 1)][g + (e >> 1) * 8] = acc[j][e];
  __syncthreads();
  constexpr int ROWS = KIND == KIND_8 ? 8 : 16;
  for (int i = threadIdx.x; i < NT * 8 * COLS; i += 32 * kWarps) {
    const int m = i / COLS, c = i % COLS, n = n0 + c;
    if (m >= p.M || n >= p.N) continue;
    float s = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      s += part[w][m][c];
      if (KIND == KIND_GATED) s2 += part[w][m][(c + 8) % ROWS];
    }
    if (p.bias) s += __bfloat162float(p.bias[n]);
    if constexpr (KIND == KIND_GATED) {
      if (p.bias) s2 += __bfloat162float(p.bias[p.N + n]);
      const float a = p.gate == EPD_GATE_SILU        ? gate_act_fast<EPD_GATE_SILU>(s)
                      : p.gate == EPD_GATE_GELU_TANH ? gate_act_fast<EPD_GATE_GELU_TANH>(s)
                                                     : gate_act_fast<EPD_GATE_GELU_ERF>(s);
      p.out[m * p.ldo + n] = __float2bfloat16_rn(a * s2);
      if (p.pre) {
        p.pre[m * p.ldp + n] = __float2bfloat16_rn(s);
        p.pre[m * p.ldp + p.N + n] = __float2bfloat16_rn(s2);
      }
    } else if (p.out_f32) {
      float* o = p.out_f32 + m * p.ldo + n;
      *o = p.accumulate ? *o + s : s;
    } else {
      p.out[m * p.ldo + n] = __float2bfloat16_rn(s);
    }
  }
}

template <int KIND>
cudaError_t launch(const FewRows& p, cudaStream_t s) {
  constexpr int COLS = KIND == KIND_16 ? 16 : 8;
  const dim3 grid((unsigned)((p.N + COLS - 1) / COLS)), block(32 * kWarps);
  if (p.M <= 8) return launch_pdl(few_rows_kernel<KIND, 1>, grid, block, 0, s, p);
  if (p.M <= 16) return launch_pdl(few_rows_kernel<KIND, 2>, grid, block, 0, s, p);
  return launch_pdl(few_rows_kernel<KIND, 4>, grid, block, 0, s, p);
}

}  // namespace

cudaError_t gated_few_rows(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                           void* pre, int64_t ldp, int64_t M, int64_t N, int64_t K, int gate, cudaStream_t s) {
  FewRows p = {};
  p.x = static_cast<const __nv_bfloat16*>(x); p.ldx = ldx;
  p.w = static_cast<const __nv_bfloat16*>(w); p.ldw = ldw;
  p.bias = static_cast<const __nv_bfloat16*>(bias);
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.out = static_cast<__nv_bfloat16*>(out); p.ldo = ldo;
  p.pre = static_cast<__nv_bfloat16*>(pre); p.ldp = ldp;
  p.gate = gate;
  return launch<KIND_GATED>(p, s);
}

cudaError_t linear_few_rows(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                            int64_t M, int64_t N, int64_t K, int flags, bool behind_gated, cudaStream_t s) {
  FewRows p = {};
  p.x = static_cast<const __nv_bfloat16*>(x); p.ldx = ldx;
  p.w = static_cast<const __nv_bfloat16*>(w); p.ldw = ldw;
  p.bias = static_cast<const __nv_bfloat16*>(bias);
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.ldo = ldo;
  if (flags & (EPD_LINEAR_ACCUMULATE | EPD_LINEAR_OUT_F32)) p.out_f32 = static_cast<float*>(out);
  else p.out = static_cast<__nv_bfloat16*>(out);
  p.accumulate = (flags & EPD_LINEAR_ACCUMULATE) != 0;
  p.weights_settled = behind_gated;
  // 8 columns a block where 16 would leave SMs without one
  return (N + 15) / 16 >= 2 * 148 ? launch<KIND_16>(p, s) : launch<KIND_8>(p, s);
}

}  // namespace epd
