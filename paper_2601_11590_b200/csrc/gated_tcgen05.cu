// The products of the gated feed-forward block and of the gradients on the 5th-generation tensor cores (bf16 operands,
// float sums), on CTA pairs with 256 x 256 accumulator tiles (tcgen05.mma.cta_group::2: each CTA stages its 128 rows of A and
// half of the B tile):
//   GATE       A = x [M, K], B = w [2N, K], both contraction-contiguous.  The pair's first CTA stages 128 gate rows of w, the
//              second the 128 up rows of the same columns, so that a thread of the epilogue holds both projections of
//              its 128 output columns: act(g) * u leaves the kernel, g and u only when the gradient will need them.
//   GATE_GRAD  A = dout [M, D] contraction-contiguous, B = w_out [D, N] row-contiguous: the tile is da = dout . w_out; the
//              epilogue reads g and u and writes dg = da u act'(g), du = da act(g): da itself is never written.
//   NN         A contraction-contiguous, B row-contiguous: dx = dout . w
//   TN         both row-contiguous: dw = dout^T . x
// A row-contiguous ("MN-major") operand is staged as boxes of 64 rows x 64 contraction steps: TMA brings 128 contiguous
// bytes of 64 rows per step, 128-byte swizzled, and the tensor core transposes on the way (descriptor: 8 KB between
// boxes, 1 KB between groups of 8 steps), so no operand is ever transposed in memory.
//
// Roles per CTA (10 warps): warp 0 TMA producer, warp 1 issues the products (in the pair's first CTA) and owns tensor memory,
// warps 2..9 epilogue, two per TMEM lane quarter, each taking half of the tile's columns in steps of 32: tcgen05.ld, the
// arithmetic in float, one rounding to bf16, a 32-row x 64-byte box in 64-byte-swizzled shared memory, TMA store.  Two
// accumulators in tensor memory: a tile's epilogue runs under the next tile's products.  Ragged extents: TMA fills loads
// with zeros and clips stores.  Every wait is bounded; on expiry the kernel drains and returns.  No load is a multicast load.
#include "gated.cuh"
#include "tcgen05_common.cuh"

namespace epd {
namespace {

using namespace tc;

enum { MODE_GATE = 0, MODE_GATE_GRAD = 1, MODE_NN = 2, MODE_TN = 3 };

constexpr int BM = 128;            // rows of A per CTA (256 per pair)
constexpr int BN = 256;            // accumulator columns
constexpr int BK = 64;             // contraction steps per stage: 128 bytes
constexpr int kEpiWarps = 8;
constexpr int kThreads = 32 * (2 + kEpiWarps);
constexpr int kTileBytes = BM * BK * 2;            // one operand of one CTA: 16 KB
constexpr int kStageBytes = 2 * kTileBytes;
constexpr int kBoxBytes = 8192;                    // 64 rows x 64 steps of a row-contiguous operand
constexpr int kBufBytes = 32 * 64;                 // staged output box: 32 rows x 32 bf16

// 5 stages and 3 staged boxes per epilogue warp; GATE_GRAD, which also fetches g and u through the staged boxes ahead of
// time, has 4 stages and 3 pairs of boxes.
template <int MODE> struct Smem {
  static constexpr int kStages = MODE == MODE_GATE_GRAD ? 4 : 5;
  static constexpr int kBufs = MODE == MODE_GATE_GRAD ? 6 : 3;
  static constexpr int kBufOffset = kStages * kStageBytes;
  static constexpr int kBarOffset = kBufOffset + kEpiWarps * kBufs * kBufBytes;
  // full[S], empty[S], tmem_full[2], tmem_empty[2], drain, spare; per epilogue warp 3 fetch barriers; TMEM base, abort flag
  static constexpr int kFetchOffset = kBarOffset + (2 * kStages + 6) * 8;
  static constexpr int kBiasOffset = kFetchOffset + kEpiWarps * 3 * 8 + 16;
  static constexpr int kTotal = kBiasOffset + (MODE == MODE_GATE ? kEpiWarps * 128 * 4 : 0);
  static constexpr int kDynamic = kTotal + 1024;
  static_assert(kDynamic <= 232448, "exceeds the shared memory of one CTA");
  static_assert(kDynamic > 116 * 1024, "one CTA per SM is assumed by the TMEM allocation");
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t smem_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Relaxed: says only that this warp's tcgen05.ld of the accumulator have completed.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ uint64_t l2_policy(bool keep, bool normal) {
  uint64_t p;
  if (keep) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  else if (normal) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
// Load whose bytes are counted on a barrier that may live in the pair's other CTA (its cluster-window address).
__device__ __forceinline__ void tma_load_pair(void* smem_dst, const CUtensorMap* tm, int x, int y, uint32_t bar,
                                              uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%3, %4}], [%2], %5;"
      ::"r"(smem_u32(smem_dst)), "l"(tm), "r"(bar), "r"(x), "r"(y), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* smem_result, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem_result)),
               "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void umma_pair(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_both(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
      ::"r"(smem_u32(bar)), "h"((uint16_t)3)
      : "memory");
}
// bf16 x bf16 -> float, M = 256 over the pair, N = BN; a_mn / b_mn: operand row-contiguous.
__host__ __device__ constexpr uint32_t instr_desc(bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
}
// Descriptor of a staged row-contiguous operand (two boxes of 64 rows): 128-byte swizzle, kBoxBytes between boxes, 1024
// bytes between groups of 8 contraction steps.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFF) >> 4);
  d |= (uint64_t)(kBoxBytes >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Order of the output tiles.  The operand of a band of tile rows (or tile columns) stays in L2 while the other one streams
// past once per band.
struct Order {
  int by_rows, group, stream_normal;
};
__device__ __forceinline__ void tile_coords(int tile, int m_tiles, int n_tiles, const Order& o, int& mt, int& nt) {
  const int across = o.by_rows ? n_tiles : m_tiles, along = o.by_rows ? m_tiles : n_tiles;
  const int per = o.group * across, band = tile / per, r = tile - band * per;
  const int first = band * o.group, width = min(o.group, along - first);
  const int c = r / width, w = first + (r - c * width);
  mt = o.by_rows ? w : c;
  nt = o.by_rows ? c : w;
}

struct Maps {
  CUtensorMap a, b;
  CUtensorMap o0, o1, o2;      // GATE: out, g, u; GATE_GRAD: dg, du; else out
  CUtensorMap l0, l1;          // GATE_GRAD: g, u
};
struct Problem {
  int M, N, K;                 // N: columns of an output matrix
  int save_pre;                // GATE: g and u are written
  const __nv_bfloat16* bias;   // GATE: [2N] or NULL
  Order order;
  long long wait_limit;
  int* status;
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&v);
}
// One lane's row of a staged box: 16-byte piece j of row r lives at piece j ^ ((r / 2) % 4) (64-byte swizzle).
__device__ __forceinline__ uint8_t* box_piece(uint8_t* buf, int lane, int j) {
  return buf + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4);
}

template <int MODE, int GATE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
gated_pair_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Problem p) {
  using L = Smem<MODE>;
  constexpr int STAGES = L::kStages;
  constexpr bool A_MN = MODE == MODE_TN, B_MN = MODE != MODE_GATE;
  constexpr int TILE_COLS = MODE == MODE_GATE ? BN / 2 : BN;     // output columns of a tile
  constexpr int kSteps = TILE_COLS / 2 / 32;                     // 32-column steps of an epilogue warp

  pdl_launch_dependents();
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBarOffset);   // used in the leader only
  uint64_t* empty = full + STAGES;                                      // one set per CTA
  uint64_t* tmem_full = empty + STAGES;                                 // one set per CTA
  uint64_t* tmem_empty = tmem_full + 2;                                 // used in the leader only
  uint64_t* drain_bar = tmem_empty + 2;
  uint64_t* fetch = reinterpret_cast<uint64_t*>(smem + L::kFetchOffset);
  uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(fetch + kEpiWarps * 3);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_base_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const WaitCtx wc{abort_flag, map_to_rank(smem_u32(const_cast<int*>(abort_flag)), rank ^ 1u), p.wait_limit};
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int m_tiles = (p.M + 2 * BM - 1) / (2 * BM), n_tiles = (p.N + TILE_COLS - 1) / TILE_COLS;
  const int num_tiles = m_tiles * n_tiles;
  const int k_blocks = (p.K + BK - 1) / BK;
  uint32_t loads_issued = 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&tmem_full[a], 1); mbar_init(&tmem_empty[a], 2 * kEpiWarps); }
    for (int i = 0; i < kEpiWarps * 3; ++i) mbar_init(&fetch[i], 1);
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc_pair(tmem_base_slot, 2 * BN);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_slot;
  pdl_wait();   // nothing above touches global memory

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (both CTAs)
    if (lane == 0) {
      prefetch_map(&maps.a);
      prefetch_map(&maps.b);
    }
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    const uint64_t pol_a = l2_policy(p.order.by_rows, p.order.stream_normal);
    const uint64_t pol_b = l2_policy(!p.order.by_rows, p.order.stream_normal);
    for (int tile = pair; tile < num_tiles && ok; tile += n_pairs) {
      int mt, nt;
      tile_coords(tile, m_tiles, n_tiles, p.order, mt, nt);
      const int m0 = mt * (2 * BM) + (int)rank * BM;
      // this CTA's half of the B tile; GATE: gate rows in the first CTA, up rows in the second
      const int n0 = MODE == MODE_GATE ? nt * TILE_COLS + (int)rank * p.N : nt * BN + (int)rank * (BN / 2);
      for (int kb = 0; kb < k_blocks; ++kb) {
        if (!mbar_wait_warp<true>(&empty[stage], phase ^ 1, wc)) { ok = false; break; }
        uint8_t* sa = smem + stage * kStageBytes;
        uint8_t* sb = sa + kTileBytes;
        const uint32_t bar = map_to_rank(smem_u32(&full[stage]), 0);
        if (elect_one()) {
          if (rank == 0) mbar_expect_tx(&full[stage], 2 * kStageBytes);   // both CTAs' bytes
          if constexpr (A_MN) {
            tma_load_pair(sa, &maps.a, m0, kb * BK, bar, pol_a);
            tma_load_pair(sa + kBoxBytes, &maps.a, m0 + 64, kb * BK, bar, pol_a);
          } else {
            tma_load_pair(sa, &maps.a, kb * BK, m0, bar, pol_a);
          }
          if constexpr (B_MN) {
            tma_load_pair(sb, &maps.b, n0, kb * BK, bar, pol_b);
            tma_load_pair(sb + kBoxBytes, &maps.b, n0 + 64, kb * BK, bar, pol_b);
          } else {
            tma_load_pair(sb, &maps.b, kb * BK, n0, bar, pol_b);
          }
        }
        __syncwarp();
        ++loads_issued;
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ issues the products (leader only)
    if (rank == 0) {
      constexpr uint32_t idesc = instr_desc(A_MN, B_MN);
      // 16 contraction steps: 32 bytes inside a swizzled row, or two groups of 8 steps of 1024 bytes (descriptor units of 16)
      constexpr uint32_t a_step = A_MN ? 2048 / 16 : 2, b_step = B_MN ? 2048 / 16 : 2;
      int stage = 0;
      uint32_t phase = 0;
      int acc = 0;
      uint32_t acc_phase = 0;
      bool ok = true;
      for (int tile = pair; tile < num_tiles && ok; tile += n_pairs) {
        if (!mbar_wait_warp<true>(&tmem_empty[acc], acc_phase ^ 1, wc)) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * BN;
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!mbar_wait_warp<true>(&full[stage], phase, wc)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = smem_u32(smem + stage * kStageBytes);
          const uint64_t da = A_MN ? smem_desc_mn_sw128(sa) : smem_desc_k_sw128(sa);
          const uint64_t db = B_MN ? smem_desc_mn_sw128(sa + kTileBytes) : smem_desc_k_sw128(sa + kTileBytes);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < BK / 16; ++k) umma_pair(d_tmem, da + a_step * k, db + b_step * k, idesc, (kb | k) != 0);
            umma_commit_both(&empty[stage]);
          }
          __syncwarp();
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if (elect_one()) umma_commit_both(&tmem_full[acc]);
        __syncwarp();
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ epilogue (both CTAs)
    const int q = warp & 3;                          // TMEM lane quarter this warp may read
    const int half = (warp - 2) >> 2;                // which half of the columns
    uint8_t* bufs = smem + L::kBufOffset + (warp - 2) * L::kBufs * kBufBytes;
    uint64_t* fbar = fetch + (warp - 2) * 3;
    float* bs = reinterpret_cast<float*>(smem + L::kBiasOffset) + (warp - 2) * 128;   // GATE: 64 gate, 64 up
    const uint32_t tmem_empty_leader = map_to_rank(smem_u32(&tmem_empty[0]), 0);
    if (lane == 0) prefetch_map(&maps.o0);
    int acc = 0;
    uint32_t acc_phase = 0;
    uint32_t step = 0;                               // steps done by this warp over all its tiles
    uint32_t fetched = 0;                            // GATE_GRAD: steps whose g and u have been asked for
    // GATE_GRAD: asks for g and u of step c of the tile at (row, column)
    auto fetch_pre = [&](int row, int col) {
      if (lane == 0) {
        uint64_t* b = &fbar[fetched % 3];
        uint8_t* to = bufs + (fetched % 3) * 2 * kBufBytes;
        mbar_expect_tx(b, 2 * kBufBytes);
        tma_load_2d(to, &maps.l0, col, row, b);
        tma_load_2d(to + kBufBytes, &maps.l1, col, row, b);
      }
      __syncwarp();
      ++fetched;
    };
    auto origin = [&](int tile, int& row0, int& n0) {
      int mt, nt;
      tile_coords(tile, m_tiles, n_tiles, p.order, mt, nt);
      row0 = mt * (2 * BM) + (int)rank * BM + q * 32;
      n0 = nt * TILE_COLS + half * (TILE_COLS / 2);
    };
    if constexpr (MODE == MODE_GATE_GRAD) {
      if (pair < num_tiles) {
        int row0, n0;
        origin(pair, row0, n0);
        fetch_pre(row0, n0);
      }
    }
    for (int tile = pair; tile < num_tiles; tile += n_pairs) {
      int row0, n0;
      origin(tile, row0, n0);
      if constexpr (MODE == MODE_GATE) {
        __syncwarp();
        for (int i = lane; i < 128; i += 32) {
          const int col = n0 + (i & 63);
          bs[i] = p.bias != nullptr && col < p.N ? __bfloat162float(p.bias[(i >> 6) * (int64_t)p.N + col]) : 0.0f;
        }
        __syncwarp();
      }
      if (!mbar_wait_warp<true>(&tmem_full[acc], acc_phase, wc)) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + acc * BN + half * (TILE_COLS / 2) + ((uint32_t)(q * 32) << 16);
      bool ok = true;
#pragma unroll 1
      for (int c = 0; c < kSteps; ++c, ++step) {
        const int col = n0 + c * 32;
        const bool inside = row0 < p.M && col < p.N;
        if constexpr (MODE == MODE_GATE) {
          uint32_t g[32], u[32];
          tmem_ld32(taddr + c * 32, g);
          tmem_ld32(taddr + BN / 2 + c * 32, u);
          tmem_ld_wait();
          if (c == kSteps - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + acc * 8);
          }
          if (lane == 0) bulk_wait_read<0>();       // the boxes' last stores have left shared memory
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t o4[4], g4[4], u4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = 8 * j + 2 * e;
              const float2 bg = *reinterpret_cast<const float2*>(bs + c * 32 + i);
              const float2 bu = *reinterpret_cast<const float2*>(bs + 64 + c * 32 + i);
              const float g0 = __uint_as_float(g[i]) + bg.x, g1 = __uint_as_float(g[i + 1]) + bg.y;
              const float u0 = __uint_as_float(u[i]) + bu.x, u1 = __uint_as_float(u[i + 1]) + bu.y;
              o4[e] = pack2(gate_act_fast<GATE>(g0) * u0, gate_act_fast<GATE>(g1) * u1);
              g4[e] = pack2(g0, g1);
              u4[e] = pack2(u0, u1);
            }
            *reinterpret_cast<uint4*>(box_piece(bufs, lane, j)) = make_uint4(o4[0], o4[1], o4[2], o4[3]);
            if (p.save_pre) {
              *reinterpret_cast<uint4*>(box_piece(bufs + kBufBytes, lane, j)) = make_uint4(g4[0], g4[1], g4[2], g4[3]);
              *reinterpret_cast<uint4*>(box_piece(bufs + 2 * kBufBytes, lane, j)) = make_uint4(u4[0], u4[1], u4[2], u4[3]);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (inside) {
              tma_store_2d(&maps.o0, col, row0, bufs);
              if (p.save_pre) {
                tma_store_2d(&maps.o1, col, row0, bufs + kBufBytes);
                tma_store_2d(&maps.o2, col, row0, bufs + 2 * kBufBytes);
              }
            }
            bulk_commit();
          }
        } else if constexpr (MODE == MODE_GATE_GRAD) {
          // the next step's g and u: into the pair of boxes whose store was issued two steps ago
          int next_row = row0, next_col = col + 32;
          bool more = true;
          if (c == kSteps - 1) {
            more = tile + n_pairs < num_tiles;
            if (more) origin(tile + n_pairs, next_row, next_col);
          }
          if (more) {
            if (lane == 0) bulk_wait_read<1>();
            __syncwarp();
            fetch_pre(next_row, next_col);
          }
          uint32_t da[32];
          tmem_ld32(taddr + c * 32, da);
          tmem_ld_wait();
          if (c == kSteps - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + acc * 8);
          }
          if (!mbar_wait_warp(&fbar[step % 3], (step / 3) & 1, wc)) { ok = false; break; }
          uint8_t* gb = bufs + (step % 3) * 2 * kBufBytes;
          uint8_t* ub = gb + kBufBytes;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint4* gp = reinterpret_cast<uint4*>(box_piece(gb, lane, j));
            uint4* up = reinterpret_cast<uint4*>(box_piece(ub, lane, j));
            const uint4 gv = *gp, uv = *up;
            const uint32_t gw[4] = {gv.x, gv.y, gv.z, gv.w}, uw[4] = {uv.x, uv.y, uv.z, uv.w};
            uint32_t dg4[4], du4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 gf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&gw[e]));
              const float2 uf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&uw[e]));
              const float d0 = __uint_as_float(da[8 * j + 2 * e]), d1 = __uint_as_float(da[8 * j + 2 * e + 1]);
              float a0, s0, a1, s1;
              gate_act_slope_fast<GATE>(gf.x, &a0, &s0);
              gate_act_slope_fast<GATE>(gf.y, &a1, &s1);
              dg4[e] = pack2(d0 * uf.x * s0, d1 * uf.y * s1);
              du4[e] = pack2(d0 * a0, d1 * a1);
            }
            *gp = make_uint4(dg4[0], dg4[1], dg4[2], dg4[3]);
            *up = make_uint4(du4[0], du4[1], du4[2], du4[3]);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (inside) {
              tma_store_2d(&maps.o0, col, row0, gb);
              tma_store_2d(&maps.o1, col, row0, ub);
            }
            bulk_commit();
          }
        } else {
          uint32_t v[32];
          tmem_ld32(taddr + c * 32, v);
          tmem_ld_wait();
          if (c == kSteps - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + acc * 8);
          }
          uint8_t* buf = bufs + (step % 3) * kBufBytes;
          if (lane == 0) bulk_wait_read<2>();       // the box's store three steps ago
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2(__uint_as_float(v[8 * j + 2 * e]), __uint_as_float(v[8 * j + 2 * e + 1]));
            *reinterpret_cast<uint4*>(box_piece(buf, lane, j)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (inside) tma_store_2d(&maps.o0, col, row0, buf);
            bulk_commit();
          }
        }
      }
      if (!ok) break;
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
    if (lane == 0) {
      bulk_wait_all();
      // after an abort: boxes asked for and not waited for are still on their way
      for (uint32_t f = step; f < fetched; ++f) mbar_wait_drain(&fbar[f % 3], (f / 3) & 1);
    }
    __syncwarp();
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // A wait expired, here or in the pair's other CTA.  Every role has left its loop and issues nothing more; what was issued
    // completes by itself and is waited for: the leader's producer waits for the last load of every stage (its barriers
    // count both CTAs' bytes), a commit behind the leader's products reaches both CTAs' drain barriers, the epilogue warps
    // have waited for their stores and fetches; then a fixed pause, and the cluster barrier.
    if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, kStatusTimeout);
    if (warp == 0 && lane == 0 && rank == 0) drain_ring<true>(full, STAGES, loads_issued);
    if (warp == 1) {
      if (elect_one()) {
        if (rank == 0) umma_commit_both(drain_bar);
        mbar_wait_drain<true>(drain_bar, 0);
      }
      __syncwarp();
    }
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 2 * BN);
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
constexpr double kBandBytes = 40.0 * 1024 * 1024;      // what a band of one operand can count on in L2
constexpr double kSmallBand = 24.0 * 1024 * 1024;      // beside which the streamed operand keeps the ordinary priority

// Band order with the least modelled traffic: one operand once, the other once per band of the first.
Order choose_order(int64_t rows_a, int64_t rows_b, int64_t K, int tile_a, int tile_b) {
  const int ta = (int)((rows_a + tile_a - 1) / tile_a), tb = (int)((rows_b + tile_b - 1) / tile_b);
  const double band_a = 2.0 * tile_a * K, band_b = 2.0 * tile_b * K;
  auto bands = [](int tiles, double bytes) {
    const int cap = (int)(1.1 * kBandBytes / bytes) > 1 ? (int)(1.1 * kBandBytes / bytes) : 1;
    return (tiles + cap - 1) / cap;
  };
  const int na = bands(ta, band_a), nb = bands(tb, band_b);
  const double all_a = 2.0 * rows_a * K, all_b = 2.0 * rows_b * K;
  if (all_a + all_b * na <= all_b + all_a * nb) {
    const int g = (ta + na - 1) / na;
    return Order{1, g, g * band_a <= kSmallBand ? 1 : 0};
  }
  const int g = (tb + nb - 1) / nb;
  return Order{0, g, g * band_b <= kSmallBand ? 1 : 0};
}

// Operand maps: contraction-contiguous [rows, K], box 128 rows x 64; row-contiguous [K, rows], box 64 x 64.
bool operand_map(CUtensorMap* tm, const void* base, int64_t rows, int64_t K, int64_t ld, bool mn) {
  return mn ? make_tensor_map_2d(tm, base, K, rows, ld * 2, BK, 64, 2, CU_TENSOR_MAP_SWIZZLE_128B)
            : make_tensor_map_2d(tm, base, rows, K, ld * 2, BM, BK, 2, CU_TENSOR_MAP_SWIZZLE_128B);
}
// 32 x 32 boxes of a bf16 matrix [rows, cols], staged with the 64-byte swizzle.
bool box_map(CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t ld) {
  return make_tensor_map_2d(tm, base, rows, cols, ld * 2, 32, 32, 2, CU_TENSOR_MAP_SWIZZLE_64B);
}

template <int MODE, int GATE>
cudaError_t launch(const Maps& maps, Problem p, cudaStream_t s) {
  using L = Smem<MODE>;
  auto kern = gated_pair_kernel<MODE, GATE>;
  static PerDeviceOnce configured;
  cudaError_t e = once_per_device(configured, [&] {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic);
  });
  if (e != cudaSuccess) return e;
  constexpr int tile_cols = MODE == MODE_GATE ? BN / 2 : BN;
  const int64_t tiles = (int64_t)((p.M + 2 * BM - 1) / (2 * BM)) * ((p.N + tile_cols - 1) / tile_cols);
  if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
  // pairs that can be resident at once on this device (SMs pair up inside a GPC, so this can be below SMs / 2)
  static PerDeviceInt resident;
  int dev = 0;
  cudaGetDevice(&dev);
  const int slot = dev >= 0 && dev < 64 ? dev : 0;
  int max_pairs = resident.v[slot].load(std::memory_order_relaxed);
  if (max_pairs == 0 || slot != dev) {
    const int sms = device_sm_count();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sms / 2 * 2);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = L::kDynamic;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n <= 0) {
      (void)cudaGetLastError();
      n = sms / 2;
    }
    max_pairs = n < sms / 2 ? n : sms / 2;
    if (slot == dev) resident.v[slot].store(max_pairs, std::memory_order_relaxed);
  }
  const int avail = limited_sms(2 * max_pairs) / 2 > 0 ? limited_sms(2 * max_pairs) / 2 : 1;
  const int pairs = tiles < avail ? (int)tiles : avail;
  p.wait_limit = wait_limit_cycles();
  return launch_pdl(kern, dim3(2 * pairs), dim3(kThreads), L::kDynamic, s, maps, p);
}

bool matrix_ok(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

}  // namespace

bool gated_tc_supported(std::initializer_list<MatrixArg> matrices, std::initializer_list<int64_t> extents) {
  for (const MatrixArg& m : matrices)
    if (m.p && !matrix_ok(m.p, m.ld)) return false;
  for (int64_t e : extents)
    if (e < 8 || e % 8) return false;
  return tensor_maps_available();
}

cudaError_t gated_tc_forward(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* out, int64_t ldo,
                             void* pre, int64_t ldp, int64_t M, int64_t N, int64_t K, int gate, int* status,
                             cudaStream_t s) {
  Maps m = {};
  if (!operand_map(&m.a, x, M, K, ldx, false) || !operand_map(&m.b, w, 2 * N, K, ldw, false) ||
      !box_map(&m.o0, out, M, N, ldo))
    return cudaErrorInvalidValue;
  if (pre) {
    __nv_bfloat16* g = static_cast<__nv_bfloat16*>(pre);
    if (!box_map(&m.o1, g, M, N, ldp) || !box_map(&m.o2, g + N, M, N, ldp)) return cudaErrorInvalidValue;
  }
  Problem p = {};
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.save_pre = pre != nullptr;
  p.bias = static_cast<const __nv_bfloat16*>(bias);
  p.order = choose_order(M, 2 * N, K, 2 * BM, BN);
  p.status = status;
  if (gate == EPD_GATE_SILU) return launch<MODE_GATE, EPD_GATE_SILU>(m, p, s);
  if (gate == EPD_GATE_GELU_TANH) return launch<MODE_GATE, EPD_GATE_GELU_TANH>(m, p, s);
  return launch<MODE_GATE, EPD_GATE_GELU_ERF>(m, p, s);
}

cudaError_t gated_tc_gradient(const void* dout, int64_t lddo, const void* w_out, int64_t ldw, const void* pre, int64_t ldp,
                              void* dpre, int64_t lddp, int64_t M, int64_t N, int64_t D, int gate, cudaStream_t s) {
  Maps m = {};
  const __nv_bfloat16* g = static_cast<const __nv_bfloat16*>(pre);
  __nv_bfloat16* dg = static_cast<__nv_bfloat16*>(dpre);
  if (!operand_map(&m.a, dout, M, D, lddo, false) || !operand_map(&m.b, w_out, N, D, ldw, true) ||
      !box_map(&m.l0, g, M, N, ldp) || !box_map(&m.l1, g + N, M, N, ldp) || !box_map(&m.o0, dg, M, N, lddp) ||
      !box_map(&m.o1, dg + N, M, N, lddp))
    return cudaErrorInvalidValue;
  Problem p = {};
  p.M = (int)M; p.N = (int)N; p.K = (int)D;
  p.order = choose_order(M, N, D, 2 * BM, BN);
  if (gate == EPD_GATE_SILU) return launch<MODE_GATE_GRAD, EPD_GATE_SILU>(m, p, s);
  if (gate == EPD_GATE_GELU_TANH) return launch<MODE_GATE_GRAD, EPD_GATE_GELU_TANH>(m, p, s);
  return launch<MODE_GATE_GRAD, EPD_GATE_GELU_ERF>(m, p, s);
}

// out[M, N] = A . B with A [M, K] (or, a_mn, [K, M]) and B [K, N].
cudaError_t matmul_tc(bool a_mn, const void* a, int64_t lda, const void* b, int64_t ldb, void* out, int64_t ldo, int64_t M,
                      int64_t N, int64_t K, cudaStream_t s) {
  Maps m = {};
  if (!operand_map(&m.a, a, M, K, lda, a_mn) || !operand_map(&m.b, b, N, K, ldb, true) || !box_map(&m.o0, out, M, N, ldo))
    return cudaErrorInvalidValue;
  Problem p = {};
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.order = choose_order(M, N, K, 2 * BM, BN);
  return a_mn ? launch<MODE_TN, 0>(m, p, s) : launch<MODE_NN, 0>(m, p, s);
}

}  // namespace epd
