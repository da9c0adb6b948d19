// What the kernels of the gated feed-forward block share: the activations with their derivatives, in float.
#pragma once

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

}  // namespace epd
