// The gated block for one token and a handful of tokens (bf16): bound by reading the weights once.
//
// A column group is 8 output columns of the gated product (8 gate rows and the 8 up rows of the same columns: one 16-row
// operand tile, so a thread ends up holding both projections of its columns), or 8 or 16 output columns of the projection
// behind it.  A block walks column groups; its 8 warps share the contraction: warp w takes every eighth piece of 32 steps, so
// that the block reads contiguous stretches of its weight rows, and the warps' sums are added in shared memory, always in
// the same order.  The contraction may be taken in any order as long as both operands share it, so a thread takes 16
// contiguous bytes of a weight row and of a token's row as the fragments of two products (mma.sync, tokens as the 8-wide
// side).  Those pieces come by asynchronous copies into slots of shared memory that belong to the thread alone, several
// pieces ahead and across column groups: nothing has to be synchronised for them, and two or three blocks keep 48 to
// 120 KB of weights on their way to every SM (with the pieces in registers, 24 to 32 KB, 16 tokens of the 6B-class block took 46 + 32 us).
// tcgen05 has nothing to add here: the matrix pipe is idle most of the time either way.
// Token rows beyond the last and weight rows beyond the last are read from the last valid row; their results are not stored.
#include "gated.cuh"
#include "tcgen05_common.cuh"

namespace epd {
namespace {

constexpr int kWarps = 8;
constexpr int kChunk = 32;          // contraction steps of a warp's piece: 64 bytes of a row

// The 16 rows of a tile: 8 gate + 8 up rows; 16 rows; 8 rows and nothing; 16 in the first and 8 in the second of two tiles.
enum { KIND_GATED = 0, KIND_16 = 1, KIND_8 = 2, KIND_24 = 3 };
template <int KIND, int TILES> constexpr int kColumns = KIND == KIND_24 ? 24 : KIND == KIND_16 ? 16 * TILES : 8 * TILES;
// Whether tile i has rows in its second half.
__host__ __device__ constexpr bool whole_tile(int kind, int i) { return kind == KIND_24 ? i == 0 : kind != KIND_8; }

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
// 16 bytes to a slot of shared memory, zeros where `in` is false (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t slot, const __nv_bfloat16* p, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot), "l"(p), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 load_slot(uint32_t slot) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(slot) : "memory");
  return v;
}

// TILES 16-row tiles of weights and NT groups of 8 tokens to a step.
template <int KIND, int NT, int TILES>
struct Ring {
  static constexpr int kWeights = KIND == KIND_8 ? 1 : KIND == KIND_24 ? 3 : 2 * TILES;    // pieces of weights per step and thread
  static constexpr int kPieces = kWeights + NT;
  static constexpr int kBlocksPerSm = NT * TILES >= 8 ? 1 : NT * TILES >= 4 ? 2 : 3;
  static constexpr int kPieceBytes = 32 * kWarps * 16;
  static constexpr int kRows = 16 * TILES + 1;
  static constexpr int kPartBytes = 2 * kWarps * NT * 8 * kRows * 4;        // two sets of the warps' sums
  static constexpr int kDepth = (233472 / kBlocksPerSm - 1024 - kPartBytes) / (kPieces * kPieceBytes);
  static constexpr int kRingBytes = kDepth * kPieces * kPieceBytes;
  static constexpr int kBytes = kRingBytes + kPartBytes;
  static_assert(kDepth >= 3 && kBlocksPerSm * (kBytes + 1024) <= 233472, "the blocks of an SM");
  static_assert(KIND == KIND_8 ? TILES == 1 : KIND != KIND_24 || TILES == 2, "half a tile; one and a half");
};

template <int KIND, int NT, int TILES>
__global__ void __launch_bounds__(32 * kWarps, Ring<KIND, NT, TILES>::kBlocksPerSm)
few_rows_kernel(const FewRows p) {
  using R = Ring<KIND, NT, TILES>;
  constexpr int COLS = kColumns<KIND, TILES>;       // output columns of a group
  extern __shared__ __align__(16) uint8_t smem[];
  float* part = reinterpret_cast<float*>(smem + R::kRingBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int groups = (p.N + COLS - 1) / COLS;
  const int steps = (p.K + kWarps * kChunk - 1) / (kWarps * kChunk);       // of a column group
  const int mine = ((int)blockIdx.x < groups ? (groups - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0) * steps;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * 16;
  auto slot = [&](int depth, int piece) { return ring + (depth * R::kPieces + piece) * R::kPieceBytes; };
  // Tokens beyond the last one: their slots hold zeros and nothing is copied (copies of the last token's row by eight lanes
  // at once made one token slower than eight: 87 against 51 us).
  const __nv_bfloat16* xr[NT];
  bool token[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    token[j] = 8 * j + g < p.M;
    xr[j] = p.x + (token[j] ? (int64_t)(8 * j + g) * p.ldx + 8 * t : 0);
    if (!token[j]) {
#pragma unroll
      for (int d = 0; d < R::kDepth; ++d)
        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(slot(d, R::kWeights + j)), "r"(0u) : "memory");
    }
  }

  // The next pieces to ask for.  K is a multiple of 8: a 16-byte piece is whole or beyond the end.
  struct Cursor { int group, k; };
  auto advance = [&](Cursor& c) {
    c.k += kWarps * kChunk;
    if (c.k >= steps * kWarps * kChunk) { c.k -= steps * kWarps * kChunk; c.group += gridDim.x; }
  };
  auto ask_weights = [&](const Cursor& c, int depth) {
    const bool in = c.k + 8 * t < p.K;
    const __nv_bfloat16* w = p.w + (in ? c.k + 8 * t : 0);
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int n0 = c.group * COLS + i * (KIND == KIND_GATED ? 8 : 16);
      const int64_t r0 = min(n0 + g, p.N - 1);
      copy16(slot(depth, 2 * i), w + r0 * p.ldw, in);
      if (whole_tile(KIND, i)) {
        const int64_t r1 = KIND == KIND_GATED ? p.N + r0 : min(n0 + g + 8, p.N - 1);
        copy16(slot(depth, 2 * i + 1), w + r1 * p.ldw, in);
      }
    }
  };
  auto ask_tokens = [&](const Cursor& c, int depth) {
    const bool in = c.k + 8 * t < p.K;
#pragma unroll
    for (int j = 0; j < NT; ++j)
      if (token[j]) copy16(slot(depth, R::kWeights + j), xr[j] + (in ? c.k : -8 * t), in);
  };
  Cursor weights{(int)blockIdx.x, warp * kChunk}, tokens = weights;
  // Behind the block's own gated kernel the weights may be fetched before that kernel has finished.
  if (!p.weights_settled) pdl_wait();
#pragma unroll
  for (int d = 0; d < R::kDepth; ++d) {
    if (d < mine) ask_weights(weights, d);
    advance(weights);
  }
  if (p.weights_settled) pdl_wait();
  // From here on whatever ran in front of this kernel has completed: the next one may start and fetch its weights.
  pdl_launch_dependents();
#pragma unroll
  for (int d = 0; d < R::kDepth; ++d) {
    if (d < mine) ask_tokens(tokens, d);
    advance(tokens);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int done = 0, depth = 0, set = 0;
  for (int group = blockIdx.x; group < groups; group += gridDim.x, set ^= 1) {
    float acc[TILES][NT][4] = {};
    for (int s = 0; s < steps; ++s) {
      asm volatile("cp.async.wait_group %0;" ::"n"(R::kDepth - 1) : "memory");
      uint4 b[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) b[j] = load_slot(slot(depth, R::kWeights + j));
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const uint4 u = load_slot(slot(depth, 2 * i));
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (whole_tile(KIND, i)) v = load_slot(slot(depth, 2 * i + 1));
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          mma_16816(acc[i][j], u.x, v.x, u.y, v.y, b[j].x, b[j].y);
          mma_16816(acc[i][j], u.z, v.z, u.w, v.w, b[j].z, b[j].w);
        }
      }
      // the slots have been read (the products above needed them): the piece kDepth steps on takes their place
      if (++done + R::kDepth <= mine) {
        ask_weights(weights, depth);
        ask_tokens(weights, depth);
        advance(weights);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (++depth == R::kDepth) depth = 0;
    }
    // fragment: acc[i][j][0..1] = (weight row g of tile i, tokens 8j + 2t, + 1), acc[i][j][2..3] = (weight row g + 8, same)
    float* sums = part + set * (kWarps * NT * 8 * R::kRows);
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sums[(warp * NT * 8 + 8 * j + 2 * t + (e & 1)) * R::kRows + 16 * i + g + (e >> 1) * 8] = acc[i][j][e];
    __syncthreads();      // the other set is read by no one any more once every thread has come here
    const int n0 = group * COLS;
    for (int i = threadIdx.x; i < NT * 8 * COLS; i += 32 * kWarps) {
      const int m = i / COLS, c = i % COLS, n = n0 + c;
      if (m >= p.M || n >= p.N) continue;
      const int row = KIND == KIND_GATED ? c / 8 * 16 + c % 8 : c;
      float s = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        s += sums[(w * NT * 8 + m) * R::kRows + row];
        if (KIND == KIND_GATED) s2 += sums[(w * NT * 8 + m) * R::kRows + row + 8];
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
}

template <int KIND, int NT, int TILES>
cudaError_t launch_tokens(const FewRows& p, cudaStream_t s) {
  using R = Ring<KIND, NT, TILES>;
  auto kern = few_rows_kernel<KIND, NT, TILES>;
  static PerDeviceOnce configured;
  cudaError_t e = once_per_device(configured, [&] {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, R::kBytes);
  });
  if (e != cudaSuccess) return e;
  constexpr int COLS = kColumns<KIND, TILES>;
  const int groups = (p.N + COLS - 1) / COLS, most = R::kBlocksPerSm * limited_sms(device_sm_count());
  return launch_pdl(kern, dim3((unsigned)(groups < most ? groups : most)), dim3(32 * kWarps), R::kBytes, s, p);
}

// Every token row is read once per column group, so wide groups save that traffic and narrow ones fill the SMs.  Measured on
// 148 SMs: the gated product of 16 tokens with 16 columns a group against 8: 6.7 / 9.4 us with 269 groups (1152 x 4304), 31.9
// / 36.9 us with 800 (3200 x 12800); the projection behind it (12800 -> 3200) for 32 tokens with 32 / 16 / 8 columns a group:
// 25 / 32 / 53 us (100, 200, 400 groups), for one token with 16 / 8: 20 / 17 us.
cudaError_t launch_gated(const FewRows& p, cudaStream_t s) {
  if (p.M <= 8) return launch_tokens<KIND_GATED, 1, 1>(p, s);
  const bool wide = p.N / 16 >= 148;
  if (p.M <= 16) return wide ? launch_tokens<KIND_GATED, 2, 2>(p, s) : launch_tokens<KIND_GATED, 2, 1>(p, s);
  return wide ? launch_tokens<KIND_GATED, 4, 2>(p, s) : launch_tokens<KIND_GATED, 4, 1>(p, s);
}
// More than 8 tokens, columns enough for groups of 16 on every SM: the width with the fewest 16-byte pieces, of weights and tokens,
// on the SM that has most of them.  (12800 -> 3200, both products of the block: 24 columns a group, 134 groups, 55.9 us, 32
// columns, 100 groups, 58.7 for 16 tokens; 65.4 and 67.1 for 32.)
template <int NT>
cudaError_t launch_linear_many(const FewRows& p, cudaStream_t s) {
  if (p.N / 16 < 148) return launch_tokens<KIND_8, NT, 1>(p, s);
  auto busiest = [&](int64_t columns) {      // of 148 SMs, whatever an SM budget says: the same call always takes the same way
    return ((p.N + columns - 1) / columns + 147) / 148 * (columns / 8 + NT);
  };
  if (busiest(24) < busiest(32) && busiest(24) < busiest(16)) return launch_tokens<KIND_24, NT, 2>(p, s);
  return busiest(16) < busiest(32) ? launch_tokens<KIND_16, NT, 1>(p, s) : launch_tokens<KIND_16, NT, 2>(p, s);
}
cudaError_t launch_linear(const FewRows& p, cudaStream_t s) {
  if (p.M <= 8) return p.N / 16 >= 296 ? launch_tokens<KIND_16, 1, 1>(p, s) : launch_tokens<KIND_8, 1, 1>(p, s);
  return p.M <= 16 ? launch_linear_many<2>(p, s) : launch_linear_many<4>(p, s);
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
  return launch_gated(p, s);
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
  return launch_linear(p, s);
}

// ---- float ----------------------------------------------------------------------------------
// Plain multiply-adds, bound by reading the weights as well.  A warp has four weight rows (gated: the gate and up rows of two
// columns) and one or four tokens; its lanes take every 32nd 16-byte piece of the contraction, of which 1, 2, 4 or 8 warps of the
// block have a share each, and the lanes' sums are added by shuffles, the warps' in shared memory, always in the same order.
// More tokens are other blocks next to this one, which find the weights in L2 (in one block, with 8 or 16 tokens in registers,
// 8 tokens of a 3200 x 12800 block took 157 us for 129, 16 tokens 293 for 230).  One token of a 1152 x 4304 block takes 16 us
// (91 as plain-FMA tiles, which compute 64 rows whatever there is), 16 tokens 44 (92); of 3200 x 12800, 491 MB, 4 tokens 85.
namespace {


struct FewRowsF32 {
  const float *x, *w, *bias;
  int64_t ldx, ldw;
  int M, N, K;
  float *out, *pre;
  int64_t ldo, ldp;
  int gate, accumulate;
  int shares;               // warps that share a contraction
  int token_groups;         // blocks side by side that have the same weights for other tokens
};

constexpr int kRowsF32 = 4;

template <int TOKENS, bool GATED>
__global__ void __launch_bounds__(32 * kWarps) few_rows_f32_kernel(const FewRowsF32 p) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int COLS = GATED ? kRowsF32 / 2 : kRowsF32;      // output columns of a warp's rows
  __shared__ float part[kWarps][kRowsF32][TOKENS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int share = warp % p.shares, groups = kWarps / p.shares;
  const int64_t block = blockIdx.x / p.token_groups;
  const int m0 = (int)(blockIdx.x % p.token_groups) * TOKENS, M = min(p.M - m0, TOKENS);
  const int64_t n0 = (block * groups + warp / p.shares) * COLS;
  const float* w[kRowsF32];
#pragma unroll
  for (int r = 0; r < kRowsF32; ++r) {
    const int64_t n = min(n0 + r % COLS, (int64_t)p.N - 1);
    w[r] = p.w + (GATED && r >= COLS ? p.N + n : n) * p.ldw;
  }
  const float* x[TOKENS];
#pragma unroll
  for (int m = 0; m < TOKENS; ++m) x[m] = p.x + (m0 + (m < M ? m : 0)) * p.ldx;
  float acc[kRowsF32][TOKENS] = {};
  const int step = 128 * p.shares;
#pragma unroll (TOKENS == 1 ? 4 : 2)
  for (int k = 128 * share + 4 * lane; k < p.K; k += step) {
    float4 a[kRowsF32];
#pragma unroll
    for (int r = 0; r < kRowsF32; ++r) a[r] = __ldcs(reinterpret_cast<const float4*>(w[r] + k));
#pragma unroll
    for (int m = 0; m < TOKENS; ++m) {
      const float4 b = *reinterpret_cast<const float4*>(x[m] + k);
#pragma unroll
      for (int r = 0; r < kRowsF32; ++r)
        acc[r][m] = fmaf(a[r].x, b.x, fmaf(a[r].y, b.y, fmaf(a[r].z, b.z, fmaf(a[r].w, b.w, acc[r][m]))));
    }
  }
#pragma unroll
  for (int r = 0; r < kRowsF32; ++r)
#pragma unroll
    for (int m = 0; m < TOKENS; ++m) {
      float v = acc[r][m];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) part[warp][r][m] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < groups * COLS * TOKENS; i += 32 * kWarps) {
    const int c = i % COLS, m = i / COLS % TOKENS, group = i / (COLS * TOKENS);
    const int64_t n = (block * groups + group) * COLS + c, row = m0 + m;
    if (m >= M || n >= p.N) continue;
    float s = 0.0f, u = 0.0f;
    for (int k = 0; k < p.shares; ++k) {
      s += part[group * p.shares + k][c][m];
      if (GATED) u += part[group * p.shares + k][COLS + c][m];
    }
    if (p.bias) s += p.bias[n];
    if constexpr (GATED) {
      if (p.bias) u += p.bias[p.N + n];
      p.out[row * p.ldo + n] = gate_act(p.gate, s) * u;
      if (p.pre) {
        p.pre[row * p.ldp + n] = s;
        p.pre[row * p.ldp + p.N + n] = u;
      }
    } else {
      float* o = p.out + row * p.ldo + n;
      *o = p.accumulate ? *o + s : s;
    }
  }
}

template <int TOKENS, bool GATED>
cudaError_t launch_f32(FewRowsF32& p, cudaStream_t s) {
  constexpr int COLS = GATED ? kRowsF32 / 2 : kRowsF32;
  // as many warps to a contraction as fill the SMs twice, each with a whole step at least
  const int64_t warps = (p.N + COLS - 1) / COLS;
  p.token_groups = (p.M + TOKENS - 1) / TOKENS;
  p.shares = 1;
  while (p.shares < kWarps && warps * p.shares < 2 * 148 * kWarps && p.K >= 256 * p.shares) p.shares *= 2;
  const int64_t blocks = (warps * p.shares + kWarps - 1) / kWarps * p.token_groups;
  return launch_pdl(few_rows_f32_kernel<TOKENS, GATED>, dim3((unsigned)blocks), dim3(32 * kWarps), 0, s, p);
}
template <bool GATED>
cudaError_t launch_f32(FewRowsF32& p, cudaStream_t s) {
  if (p.M == 1) return launch_f32<1, GATED>(p, s);
  return launch_f32<4, GATED>(p, s);
}

}  // namespace

cudaError_t few_rows_float(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                           void* pre, int64_t ldp, int64_t M, int64_t N, int64_t K, int gate, bool accumulate, cudaStream_t s) {
  FewRowsF32 p = {};
  p.x = static_cast<const float*>(x); p.ldx = ldx;
  p.w = static_cast<const float*>(w); p.ldw = ldw;
  p.bias = static_cast<const float*>(bias);
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.out = static_cast<float*>(out); p.ldo = ldo;
  p.pre = static_cast<float*>(pre); p.ldp = ldp;
  p.gate = gate;
  p.accumulate = accumulate;
  return gate >= 0 ? launch_f32<true>(p, s) : launch_f32<false>(p, s);
}

}  // namespace epd
