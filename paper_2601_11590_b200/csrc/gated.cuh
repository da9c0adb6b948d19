// What the kernels of the gated feed-forward block share: the activations with their derivatives, in float, and the
// entry points of the tensor-core kernels.
#pragma once

#include <initializer_list>

#include "common.cuh"

namespace epd {

// act(g) with the library's accurate functions: the float path.
__device__ __forceinline__ float gate_act(int gate, float g) {
  if (gate == EPD_GATE_SILU) return g / (1.0f + expf(-g));
  if (gate == EPD_GATE_GELU_TANH) return gelu_tanh_f(g);
  return 0.5f * g * erfcf(-0.7071067811865476f * g);
}

// act(g) and act'(g).  Where an intermediate could leave the range of float (the cube of a large g, or the
// difference 1 - s times an infinite factor) the correction term is formed from g held to [-20, 20], beyond which
// it is zero in float anyway.
__device__ __forceinline__ void gate_act_slope(int gate, float g, float* act, float* slope) {
  const float c = fminf(fmaxf(g, -20.0f), 20.0f);
  if (gate == EPD_GATE_SILU) {
    const float s = 1.0f / (1.0f + expf(-g));
    *act = g * s;
    *slope = s * (1.0f + g * (1.0f / (1.0f + expf(g))));       // 1 - s without cancellation
  } else if (gate == EPD_GATE_GELU_TANH) {
    const float k = 0.7978845608028654f;
    const float t = tanhf(k * (g + 0.044715f * g * g * g)), tc = tanhf(k * (c + 0.044715f * c * c * c));
    *act = 0.5f * g * (1.0f + t);
    *slope = 0.5f * (1.0f + t) + 0.5f * c * (1.0f - tc * tc) * k * (1.0f + 0.134145f * c * c);
  } else {
    const float phi = 0.5f * erfcf(-0.7071067811865476f * g);
    *act = g * phi;
    *slope = phi + c * expf(-0.5f * c * c) * 0.3989422804014327f;
  }
}

// The same behind bf16 results: sigmoid and exponential from the special-function unit (relative error 2^-21, far
// inside the rounding to bf16).  tanh-GELU as x * sigmoid(2 z), which is the same function: 0.5 (1 + tanh z) = sigmoid(2 z).
__device__ __forceinline__ float sigmoid_fast(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return r;
}
// Phi(x), with the rational approximation 7.1.26 of Abramowitz & Stegun's handbook (absolute error 1.5e-7), and
// exp(-x^2 / 2).
__device__ __forceinline__ float normal_cdf_fast(float x, float* gauss) {
  const float z = fabsf(x) * 0.70710678118654752f;
  float t, e;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(0.3275911f, z, 1.0f)));
  float poly = fmaf(1.061405429f, t, -1.453152027f);
  poly = fmaf(poly, t, 1.421413741f);
  poly = fmaf(poly, t, -0.284496736f);
  poly = fmaf(poly, t, 0.254829592f);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * z * -1.4426950408889634f));
  *gauss = e;
  const float tail = 0.5f * poly * t * e;
  return x < 0.0f ? tail : 1.0f - tail;
}

template <int GATE>
__device__ __forceinline__ float gate_act_fast(float g) {
  if constexpr (GATE == EPD_GATE_SILU) return g * sigmoid_fast(g);
  if constexpr (GATE == EPD_GATE_GELU_TANH) return g * sigmoid_fast(1.5957691216057308f * (g + 0.044715f * g * g * g));
  float e;
  return g * normal_cdf_fast(g, &e);
}

// The correction term is formed from g held to a range outside of which it is zero: see gate_act_slope().
template <int GATE>
__device__ __forceinline__ void gate_act_slope_fast(float g, float* act, float* slope) {
  if constexpr (GATE == EPD_GATE_SILU) {
    const float s = sigmoid_fast(g);
    *act = g * s;
    *slope = fmaf(*act, 1.0f - s, s);
  } else if constexpr (GATE == EPD_GATE_GELU_TANH) {
    const float c = fminf(fmaxf(g, -10.0f), 10.0f);
    const float s = sigmoid_fast(1.5957691216057308f * (g + 0.044715f * g * g * g));
    *act = g * s;
    *slope = fmaf(c * s * (1.0f - s), 1.5957691216057308f * fmaf(0.134145f * c, c, 1.0f), s);
  } else {
    const float c = fminf(fmaxf(g, -20.0f), 20.0f);
    float e;
    const float phi = normal_cdf_fast(g, &e);
    *act = g * phi;
    *slope = fmaf(c * 0.3989422804014327f, e, phi);
  }
}

// ---- tensor-core kernels (gated_tcgen05.cu) ---------------------------------------------------
struct MatrixArg {
  const void* p;
  int64_t ld;
};
// Every matrix on a 16-byte boundary with a leading dimension that is a multiple of 8 (NULL ones do not count), every
// extent a multiple of 8.
bool gated_tc_supported(std::initializer_list<MatrixArg> matrices, std::initializer_list<int64_t> extents);
cudaError_t gated_tc_forward(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                             void* pre, int64_t ldp, int64_t M, int64_t N, int64_t K, int gate, cudaStream_t s);
// sums: [ceil(M / 32), 2N] floats, the column sums of every 32 rows of dpre, or NULL.
cudaError_t gated_tc_gradient(const void* dout, int64_t lddo, const void* w_out, int64_t ldw, const void* pre, int64_t ldp,
                              void* dpre, int64_t lddp, float* sums, int64_t M, int64_t N, int64_t D, int gate,
                              cudaStream_t s);
// A float matrix [rows, cols] as three bf16 planes of plane_rows rows (a multiple of 64, zeros behind the last row), one below
// the other, leading dimension ld (a multiple of 8).
struct Planes {
  __nv_bfloat16* p;
  int64_t plane_rows, cols, ld;
};
struct PlaneArg {
  const float* src;          // NULL: left out
  int64_t ld, rows;
  Planes planes;
};
cudaError_t split_planes(std::initializer_list<PlaneArg> list, cudaStream_t s);     // up to five
// The products of float matrices given as planes.  out_planes: the planes of `out` are written too.
cudaError_t gated_f32_forward(const Planes& x, const Planes& w, const void* bias, float* out, int64_t ldo, float* pre,
                              int64_t ldp, const Planes* out_planes, int64_t M, int64_t N, int64_t K, int gate,
                              cudaStream_t s);
cudaError_t gated_f32_gradient(const Planes& dout, const Planes& w_out, const float* pre, int64_t ldp, const Planes& dpre,
                               float* sums, int64_t M, int64_t N, int64_t D, int gate, cudaStream_t s);
cudaError_t linear_f32(const Planes& x, const Planes& w, const void* bias, float* out, int64_t ldo, int64_t M, int64_t N,
                       int64_t K, bool accumulate, cudaStream_t s);
// out[M, N] = A . B with A [M, K] (or, a_mn, [K, M]) and B [K, N], all bf16 or all float; out NULL: not formed, but planned for.
struct ProductArg {
  const void* a;
  int64_t lda;
  bool a_mn;
  const void* b;
  int64_t ldb;
  void* out;
  int64_t ldo;
  int64_t M, N, K;
  const Planes *planes_a, *planes_b;   // float matrices (out too): in place of a and b
};
// Up to three products that do not depend on one another.
cudaError_t matmul_tc_group(const ProductArg* list, int n, cudaStream_t s);
// A linear layer (bias or NULL; EPD_LINEAR_ACCUMULATE / EPD_LINEAR_OUT_F32) whose tiles are too few for the machine, the
// contraction of every tile shared among the pairs of a cluster.  Only where linear_tc_split_pays().
bool linear_tc_split_pays(int64_t M, int64_t N, int64_t K);
cudaError_t linear_tc_split(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                            int64_t M, int64_t N, int64_t K, int flags, cudaStream_t s);

// ---- one token to kFewRows tokens (gated_few_rows.cu) -------------------------------------------
constexpr int kFewRows = 32;
cudaError_t gated_few_rows(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                           void* pre, int64_t ldp, int64_t M, int64_t N, int64_t K, int gate, cudaStream_t s);
// out[M, N] = x . w^T + bias; flags EPD_LINEAR_ACCUMULATE / EPD_LINEAR_OUT_F32.  behind_gated: the kernel in front on the
// stream is gated_few_rows.
cudaError_t linear_few_rows(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                            int64_t M, int64_t N, int64_t K, int flags, bool behind_gated, cudaStream_t s);

}  // namespace epd
