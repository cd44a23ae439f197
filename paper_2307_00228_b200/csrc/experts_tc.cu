// The products of it_experts_forward on the tensor cores: one persistent, warp-specialised kernel over tiles of 128 places of one expert,
//   D[128, cols] = A[places, K] * W[expert][K, cols]
// with tcgen05.mma (accumulators in TMEM, two of them, so that a tile's epilogue runs beside the next tile's products), operands
// staged by TMA in 128-byte-swizzled k-blocks.  The rows of A are fetched where they lie, four to a copy (tile::gather4), by the place's
// vertex; the weights are taken as they are, [K, columns], which makes B an MN-major operand, so nothing is transposed or prepared.
// bf16 (kind::f16), e4m3 (kind::f8f6f4), and fp32 as three bf16 parts a value in six products per k-block, the smallest first
// (what is left out is 2^-24 of a term).
//
// Every wait on an mbarrier is bounded: when one gives up, the CTA raises a flag that all roles poll, waits for its copies and products in
// flight, frees its TMEM and returns, and a status word in global memory is set.
#include "experts.cuh"
#include "tc.cuh"

namespace {

constexpr int EX_EPI_WARPS = 8;   // two per TMEM lane quarter, each takes every other chunk of columns
constexpr int EX_TMA_WARPS = 4;   // each fetches a quarter of a tile's rows: a copy of four rows takes some 50 cycles to issue
constexpr int EX_EPI_WARP0 = EX_TMA_WARPS + 1;
constexpr int EX_THREADS = 32 * (EX_EPI_WARP0 + EX_EPI_WARPS);   // warps 0-3 TMA, warp 4 MMA + TMEM, warps 5-12 epilogue
constexpr int EX_STAGE_A = TC_BM * TC_KBLOCK_BYTES;
constexpr int EX_STAGING = 2048;   // per epilogue warp: 32 rows of 64 bytes (of 128 bytes they would cost a stage of operands)
constexpr int EX_CONSTS = 2 * 128 * 4;   // per epilogue warp: bias and scale of its columns
constexpr int EX_MAX_STAGES = 8;
constexpr int EX_EPI_BACKOFF = 64, EX_TMA_BACKOFF = 32;   // ns between polls

__device__ __forceinline__ void tma_gather4(void *dst, const CUtensorMap *map, int c, const int4 &rows, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c), "r"(rows.x), "r"(rows.y), "r"(rows.z), "r"(rows.w)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int c0, int c1, int c2, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// Descriptor of an MN-major tile: panels of 128 bytes of columns x the k-block's rows (128 bytes apart, swizzled), `panel` bytes each.
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t smem_addr, uint32_t panel) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(panel >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
template <bool EIGHT>
__device__ __forceinline__ void ex_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (EIGHT) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
  } else {
    tc_mma<false>(d_tmem, a_desc, b_desc, idesc, accumulate);
  }
}

__device__ __forceinline__ void expert_act(float (&v)[16], int act) {
  if (act == IT_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaxf(v[i], 0.f);
  } else if (act != IT_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = it_expert_act(v[i], act);
  }
}

struct ExParams {
  const int32_t *order, *tile_expert, *n_tiles;
  int tiles_max;
  int n_splits, bn, cols_per_tile;   // column tiles; columns of an accumulator; columns of the result in a tile (gated: bn / 2)
  int K, kb, passes;                 // k-blocks of a pass; passes: 1, or the six products of fp32 parts
  int stages;
  int gather_div;                    // > 0: row of A = place / gather_div; 0: row = position
  int a_rows;                        // rows of one part of A
  int n_experts, w_cols, cols, act, gated;
  const float *bias, *w_scale, *x_scale, *weights;
  int x_div;                         // place / x_div = vertex (for x_scale)
  void *dst;
  int64_t part_stride;               // elements from one part of the result to the next
  int *status;
  uint32_t spin_limit;
  int no_loads;
};

// the parts of A and W that pass i multiplies, smallest products first
__device__ __forceinline__ void pass_parts(int passes, int i, int *pa, int *pb) {
  constexpr uint32_t A = 0x001102u, B = 0x010120u;   // nibble i: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
  *pa = passes == 1 ? 0 : (int)((A >> (4 * i)) & 15u);
  *pb = passes == 1 ? 0 : (int)((B >> (4 * i)) & 15u);
}

template <bool EIGHT, it_expert_store STORE>
__global__ void __launch_bounds__(EX_THREADS, 1)
expert_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const ExParams p) {
  extern __shared__ unsigned char smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int BK = EIGHT ? 128 : 64;                  // elements of a k-block, and columns of a panel
  constexpr int PANEL = BK * TC_KBLOCK_BYTES;           // bytes of a panel of W: BK rows x 128 bytes
  const int b_bytes = p.bn * TC_KBLOCK_BYTES, stage_bytes = EX_STAGE_A + b_bytes;

  unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char *staging = base + (size_t)p.stages * stage_bytes;
  unsigned char *consts = staging + (STORE == IT_EXPERT_PARTS ? 0 : EX_EPI_WARPS * EX_STAGING);
  uint64_t *full = reinterpret_cast<uint64_t *>(consts + EX_EPI_WARPS * EX_CONSTS);   // [stages]
  uint64_t *empty = full + EX_MAX_STAGES;      // [stages]
  uint64_t *acc_full = empty + EX_MAX_STAGES;  // [2]
  uint64_t *acc_empty = acc_full + 2;          // [2]
  uint64_t *mma_done = acc_empty + 2;          // [1]
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 1);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  uint32_t tmem_cols = 32;
  while (tmem_cols < 2u * (uint32_t)p.bn) tmem_cols <<= 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], p.gather_div ? EX_TMA_WARPS : 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&acc_full[a], 1);
      mbar_init(&acc_empty[a], EX_EPI_WARPS);
    }
    mbar_init(mma_done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == EX_TMA_WARPS) {
    tmem_alloc(tmem_slot, tmem_cols);
    tmem_relinquish();
  }
  it_allow_next();
  it_wait_prior();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  int m_tiles = *p.n_tiles;
  m_tiles = m_tiles < p.tiles_max ? m_tiles : p.tiles_max;
  const int64_t n_tiles = (int64_t)m_tiles * p.n_splits;
  const int KB = p.kb * p.passes;

  if (warp < EX_TMA_WARPS) {
    // ------------------------------------------------------------------ TMA producers: eight lanes of a warp four rows of A each; warp 0 the weights
    uint32_t stage = 0, phase = 0;
    bool ok = !p.no_loads && (warp == 0 || p.gather_div), came_round = false;
    const uint32_t my_bytes = (p.gather_div ? EX_STAGE_A / EX_TMA_WARPS : EX_STAGE_A) + (warp == 0 ? b_bytes : 0);
    for (int64_t tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x) {
      const int m = (int)(tile / p.n_splits), c0 = (int)(tile % p.n_splits) * p.cols_per_tile;
      const int e = p.tile_expert[m];
      int4 rows = make_int4(0, 0, 0, 0);
      if (p.gather_div && lane < 8) {
        const int4 at = *reinterpret_cast<const int4 *>(p.order + (int64_t)m * TC_BM + warp * 32 + lane * 4);
        // positions of no place read the first row, and their products go nowhere
        rows.x = at.x < 0 ? 0 : at.x / p.gather_div; rows.y = at.y < 0 ? 0 : at.y / p.gather_div;
        rows.z = at.z < 0 ? 0 : at.z / p.gather_div; rows.w = at.w < 0 ? 0 : at.w / p.gather_div;
      }
      for (int pass = 0; pass < p.passes && ok; ++pass) {
        int pa, pb;
        pass_parts(p.passes, pass, &pa, &pb);
        const int row0 = pa * p.a_rows;
        const int4 r = make_int4(rows.x + row0, rows.y + row0, rows.z + row0, rows.w + row0);
        for (int kb = 0; kb < p.kb; ++kb) {
          if (lane == 0) {
            ok = mbar_wait(&empty[stage], phase ^ 1u, abort_flag, p.spin_limit, EX_TMA_BACKOFF);
            if (ok) mbar_arrive_expect_tx(&full[stage], my_bytes);
          }
          ok = __shfl_sync(0xffffffffu, (int)ok, 0);
          if (!ok) break;
          unsigned char *to = base + (size_t)stage * stage_bytes;
          if (p.gather_div && lane < 8) tma_gather4(to + (warp * 32 + lane * 4) * TC_KBLOCK_BYTES, &map_a, kb * BK, r, &full[stage]);
          if (warp == 0) {
            if (lane == 8 && !p.gather_div) tma_load_2d(to, &map_a, kb * BK, row0 + m * TC_BM, &full[stage]);
            if (lane >= 16 && lane - 16 < p.bn / BK) {   // a panel of the weights a lane
              // gated: the first half of the panels are columns of the gate, the second of what it gates
              const int c = (lane - 16) * BK, col = p.gated && c >= p.cols_per_tile ? p.cols + c0 + c - p.cols_per_tile : c0 + c;
              tma_load_3d(to + EX_STAGE_A + (lane - 16) * PANEL, &map_w, col, kb * BK, pb * p.n_experts + e, &full[stage]);
            }
          }
          if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; came_round = true; }
        }
      }
    }
    __syncwarp();
    // (after an abort a stage may be armed by some of the warps only: this wait is then one for the copies in flight by its limit)
    if (lane == 0) ring_drain(full, (uint32_t)p.stages, stage, phase, came_round);
  } else if (warp == EX_TMA_WARPS) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      // D = fp32, A K-major, B MN-major (bit 16), N = bn, M = 128; operands bf16 (1) or e4m3 (0)
      const uint32_t fmt = EIGHT ? 0u : 1u;
      const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | (1u << 16) | ((uint32_t)(p.bn >> 3) << 17) | ((uint32_t)(TC_BM >> 4) << 24);
      uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
      bool ok = true;
      for (int64_t tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x) {
        ok = mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag, p.spin_limit);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * (uint32_t)p.bn;
        for (int kb = 0; kb < KB; ++kb) {
          ok = mbar_wait(&full[stage], phase, abort_flag, p.spin_limit);
          if (!ok) break;
          tc_fence_after();
          const uint32_t a_s = smem_u32(base + (size_t)stage * stage_bytes), b_s = a_s + EX_STAGE_A;
#pragma unroll
          for (int k = 0; k < 4; ++k)   // four steps of 32 bytes of K: a quarter of the k-block's rows of W
            ex_mma<EIGHT>(d_tmem, make_desc(a_s + k * 32), make_desc_mn(b_s + k * (PANEL / 4), PANEL), idesc, (kb | k) != 0);
          tc_commit(&empty[stage]);
          if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        tc_commit(&acc_full[acc]);
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      tc_commit(mma_done);
      mbar_drain(mma_done, 0);
    }
  } else {
    // ------------------------------------------------------------------ epilogue: a thread per row of the tile, a warp per 32 rows and chunk
    const int quarter = warp & 3, sub = (warp - EX_EPI_WARP0) >> 2;   // a warp may only touch TMEM lanes [32 * (warp % 4), +32)
    constexpr bool F32_OUT = STORE == IT_EXPERT_SUMS || STORE == IT_EXPERT_OUT_F32;
    constexpr int CHUNK = F32_OUT ? 32 : 64;   // columns that a warp takes at a time: 128 bytes of a row
    const uint32_t stage_s = smem_u32(staging) + (uint32_t)(warp - EX_EPI_WARP0) * EX_STAGING, swz = ((uint32_t)lane >> 1) & 3u;
    float *bias_s = reinterpret_cast<float *>(consts + (warp - EX_EPI_WARP0) * EX_CONSTS), *scale_s = bias_s + 128;
    uint32_t acc = 0, acc_phase = 0;
    for (int64_t tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
      const int m = (int)(tile / p.n_splits), c_tile = (int)(tile % p.n_splits) * p.cols_per_tile;
      const int64_t pos0 = (int64_t)m * TC_BM + quarter * 32;
      const int place = p.order[pos0 + lane], e = p.tile_expert[m];
      const int64_t w_row = (int64_t)e * p.w_cols;
      {
        // constants of this warp's columns, four a lane, in the order in which it comes to them (gated: 64 of the gate, then 64 of what it
        // gates); loaded while the product runs (by the epilogue itself, column by column, they took four times the rest of it)
        const int l4 = lane * 4;
        const int c = c_tile + (p.gated ? sub * CHUNK + (l4 & 63) : ((l4 / CHUNK) * 2 + sub) * CHUNK + l4 % CHUNK);
        const int64_t at = w_row + c + (p.gated && l4 >= 64 ? p.cols : 0);
        float4 b = make_float4(0.f, 0.f, 0.f, 0.f), s = make_float4(1.f, 1.f, 1.f, 1.f);
        if (c < p.cols) {
          if (p.bias) b = __ldg(reinterpret_cast<const float4 *>(p.bias + at));
          if constexpr (EIGHT) s = __ldg(reinterpret_cast<const float4 *>(p.w_scale + at));
        }
        __syncwarp();   // the previous tile's have been read
        *reinterpret_cast<float4 *>(bias_s + l4) = b;
        if constexpr (EIGHT) *reinterpret_cast<float4 *>(scale_s + l4) = s;
      }
      const float xs = EIGHT && place >= 0 ? p.x_scale[place / p.x_div] : 1.f;
      const float weight = (STORE == IT_EXPERT_OUT_BF16 || STORE == IT_EXPERT_OUT_F32) && place >= 0 ? p.weights[place] : 1.f;
      const bool ok = mbar_wait(&acc_full[acc], acc_phase, abort_flag, p.spin_limit, EX_EPI_BACKOFF);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * (uint32_t)p.bn;
      int lc = 0;   // column among this warp's
      for (int ch = sub * CHUNK; ch < p.cols_per_tile && c_tile + ch < p.cols; ch += 2 * CHUNK, lc += CHUNK) {
#pragma unroll
        for (int q = 0; q < CHUNK; q += 16) {
          const int c = c_tile + ch + q;   // first column of 16 (columns past the last are computed and not stored)
          float v[16];
          auto finish = [&](int tmem_col, int at) {   // accumulator -> scaled, with the bias
            uint32_t r[16];
            tmem_ld16(taddr + (uint32_t)tmem_col, r);
            float4 b[4], s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              b[i] = *reinterpret_cast<const float4 *>(bias_s + at + 4 * i);
              if constexpr (EIGHT) s[i] = *reinterpret_cast<const float4 *>(scale_s + at + 4 * i);
            }
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if constexpr (EIGHT) {
                v[4 * i] = fmaf(__uint_as_float(r[4 * i]) * xs, s[i].x, b[i].x); v[4 * i + 1] = fmaf(__uint_as_float(r[4 * i + 1]) * xs, s[i].y, b[i].y);
                v[4 * i + 2] = fmaf(__uint_as_float(r[4 * i + 2]) * xs, s[i].z, b[i].z); v[4 * i + 3] = fmaf(__uint_as_float(r[4 * i + 3]) * xs, s[i].w, b[i].w);
              } else {
                v[4 * i] = __uint_as_float(r[4 * i]) + b[i].x; v[4 * i + 1] = __uint_as_float(r[4 * i + 1]) + b[i].y;
                v[4 * i + 2] = __uint_as_float(r[4 * i + 2]) + b[i].z; v[4 * i + 3] = __uint_as_float(r[4 * i + 3]) + b[i].w;
              }
            }
          };
          if (p.gated) {
            float gate[16];
            finish(ch + q, q);
            expert_act(v, p.act);
#pragma unroll
            for (int i = 0; i < 16; ++i) gate[i] = v[i];
            finish(p.cols_per_tile + ch + q, 64 + q);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] *= gate[i];
          } else {
            finish(ch + q, lc + q);
            expert_act(v, p.act);
          }
          if constexpr (STORE == IT_EXPERT_PARTS) {
            uint32_t w[3][8];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint32_t u = __float_as_uint(v[i]);
              const float r1 = v[i] - __uint_as_float(u & 0xffff0000u);
              const uint32_t u1 = __float_as_uint(r1), u2 = __float_as_uint(r1 - __uint_as_float(u1 & 0xffff0000u));
              if (i & 1) { w[0][i >> 1] |= u & 0xffff0000u; w[1][i >> 1] |= u1 & 0xffff0000u; w[2][i >> 1] |= u2 & 0xffff0000u; }
              else { w[0][i >> 1] = u >> 16; w[1][i >> 1] = u1 >> 16; w[2][i >> 1] = u2 >> 16; }
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) {
              uint2 *to = reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(p.dst) + k * p.part_stride + (pos0 + lane) * p.cols + c);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (place >= 0 && c + 4 * i < p.cols) to[i] = make_uint2(w[k][2 * i], w[k][2 * i + 1]);
            }
            __syncwarp();   // (the loads from TMEM are taken by whole warps)
          } else if constexpr (F32_OUT) {
            if constexpr (STORE == IT_EXPERT_OUT_F32) {
#pragma unroll
              for (int i = 0; i < 16; ++i) v[i] *= weight;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
              st_shared_v4(stage_s + (uint32_t)lane * 64u + (((uint32_t)i ^ swz) << 4), __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                           __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
          } else {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              if (STORE == IT_EXPERT_OUT_BF16) { v[2 * i] *= weight; v[2 * i + 1] *= weight; }
              const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
              w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            st_shared_v4(stage_s + (uint32_t)lane * 64u + ((((uint32_t)(q & 31) / 8) ^ swz) << 4), w[0], w[1], w[2], w[3]);
            st_shared_v4(stage_s + (uint32_t)lane * 64u + ((((uint32_t)(q & 31) / 8 + 1) ^ swz) << 4), w[4], w[5], w[6], w[7]);
          }
          if (STORE != IT_EXPERT_PARTS && (F32_OUT || (q & 16))) {
            // rows of 64 bytes out of the staging tile, four lanes a row
            __syncwarp();
            constexpr int ESIZE = F32_OUT ? 4 : 2;
            const int piece = lane & 3, c64 = c_tile + ch + (F32_OUT ? q : q - 16) + piece * (16 / ESIZE);
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 8) {
              const int r = r0 + (lane >> 2);
              const int at = __shfl_sync(0xffffffffu, place, r);
              uint4 d;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(d.x), "=r"(d.y), "=r"(d.z), "=r"(d.w)
                           : "r"(stage_s + (uint32_t)r * 64u + ((uint32_t)(piece ^ ((r >> 1) & 3)) << 4)) : "memory");
              if (at >= 0 && c64 < p.cols) {
                const int64_t row = STORE == IT_EXPERT_OUT_BF16 || STORE == IT_EXPERT_OUT_F32 ? (int64_t)at : pos0 + r;
                *reinterpret_cast<uint4 *>(reinterpret_cast<unsigned char *>(p.dst) + (row * p.cols + c64) * ESIZE) = d;
              }
            }
            __syncwarp();
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[acc]);
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.status, 1);
  if (warp == EX_TMA_WARPS) {
    tc_fence_after();
    tmem_dealloc(tmem_base, tmem_cols);
  }
}

// ----------------------------------------------------------------------------- host side
it_status encode(CUtensorMap *map, bool eight, const void *ptr, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box) {
  EncodeTiledFn enc = get_encode();
  IT_REQUIRE(enc != nullptr, IT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = enc(map, eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(ptr), dims, strides, box, estr,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  IT_REQUIRE(r == CUDA_SUCCESS, IT_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return IT_OK;
}

template <bool EIGHT, it_expert_store STORE>
it_status launch(const CUtensorMap &ma, const CUtensorMap &mw, const ExParams &p, int grid, int smem, double bytes, double flops, cudaStream_t st) {
  IT_CUDA_TRY(cudaFuncSetAttribute(expert_gemm_kernel<EIGHT, STORE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  IT_LAUNCH(IT_K_EXPERT_GEMM, bytes, flops, st, IT_CUDA_TRY(it_launch_pdl(expert_gemm_kernel<EIGHT, STORE>, dim3((unsigned)grid), dim3(EX_THREADS), smem, st, ma, mw, p)));
  return IT_OK;
}

}  // namespace

it_status it_launch_expert_gemm(const it_experts_args &a, const it_experts_plan &q, const it_expert_gemm &g, cudaStream_t st) {
  const int elem = g.eight ? 1 : 2, BK = TC_KBLOCK_BYTES / elem;
  ExParams p{};
  p.order = q.order; p.tile_expert = q.tile_expert; p.n_tiles = q.n_tiles; p.tiles_max = (int)q.tiles_max;
  p.K = g.K; p.kb = (g.K + BK - 1) / BK; p.passes = g.parts == 3 ? 6 : 1;
  p.gather_div = g.gather ? a.d.top_k : 0; p.a_rows = (int)g.a_rows;
  p.n_experts = a.d.n_experts; p.w_cols = g.w_cols; p.cols = g.cols; p.act = g.act; p.gated = g.gated;
  p.bias = g.bias; p.w_scale = g.w_scale; p.x_scale = g.x_scale; p.weights = a.weights; p.x_div = a.d.top_k;
  p.dst = g.dst; p.part_stride = q.tiles_max * TC_BM * (int64_t)g.cols; p.status = a.status;
  p.spin_limit = g.spin_limit ? g.spin_limit : TC_SPIN_LIMIT; p.no_loads = g.no_loads;
  // columns in as few tiles as 256 accumulator columns allow, of equal width in whole panels
  const int most = g.gated ? 128 : 256;
  p.n_splits = (g.cols + most - 1) / most;
  p.cols_per_tile = ((g.cols + p.n_splits - 1) / p.n_splits + BK - 1) / BK * BK;
  p.n_splits = (g.cols + p.cols_per_tile - 1) / p.cols_per_tile;
  p.bn = g.gated ? 2 * p.cols_per_tile : p.cols_per_tile;

  const cuuint64_t da[2] = {(cuuint64_t)g.K, (cuuint64_t)(g.a_rows * g.parts)}, sa[1] = {(cuuint64_t)g.K * elem};
  const cuuint32_t ba[2] = {(cuuint32_t)BK, (cuuint32_t)(g.gather ? 1 : TC_BM)};
  const cuuint64_t dw[3] = {(cuuint64_t)g.w_cols, (cuuint64_t)g.K, (cuuint64_t)a.d.n_experts * g.parts};
  const cuuint64_t sw[2] = {(cuuint64_t)g.w_cols * elem, (cuuint64_t)g.w_cols * elem * (cuuint64_t)g.K};
  const cuuint32_t bw[3] = {(cuuint32_t)BK, (cuuint32_t)BK, 1};
  CUtensorMap ma, mw;
  IT_TRY(encode(&ma, g.eight, g.A, 2, da, sa, ba));
  IT_TRY(encode(&mw, g.eight, g.W, 3, dw, sw, bw));

  const int stage = EX_STAGE_A + p.bn * TC_KBLOCK_BYTES, fixed = 1024 + (g.store == IT_EXPERT_PARTS ? 0 : EX_EPI_WARPS * EX_STAGING) + EX_EPI_WARPS * EX_CONSTS + (2 * EX_MAX_STAGES + 8) * 8;
  p.stages = (227 * 1024 - fixed) / stage;
  if (p.stages > EX_MAX_STAGES) p.stages = EX_MAX_STAGES;
  const int smem = fixed + p.stages * stage;
  const int64_t tiles = q.tiles_max * p.n_splits;
  const int grid = (int)(tiles < a.sms ? tiles : a.sms);
  const int64_t places = a.n * a.d.top_k;
  const double flops = 2.0 * places * g.K * (double)g.w_cols, bytes = (double)places * (g.K * elem * g.parts + g.cols * 4.0);
  switch (g.store) {
    case IT_EXPERT_HIDDEN: return g.eight ? launch<true, IT_EXPERT_HIDDEN>(ma, mw, p, grid, smem, bytes, flops, st) : launch<false, IT_EXPERT_HIDDEN>(ma, mw, p, grid, smem, bytes, flops, st);
    case IT_EXPERT_PARTS: return launch<false, IT_EXPERT_PARTS>(ma, mw, p, grid, smem, bytes, flops, st);
    case IT_EXPERT_SUMS: return g.eight ? launch<true, IT_EXPERT_SUMS>(ma, mw, p, grid, smem, bytes, flops, st) : launch<false, IT_EXPERT_SUMS>(ma, mw, p, grid, smem, bytes, flops, st);
    case IT_EXPERT_OUT_BF16: return g.eight ? launch<true, IT_EXPERT_OUT_BF16>(ma, mw, p, grid, smem, bytes, flops, st) : launch<false, IT_EXPERT_OUT_BF16>(ma, mw, p, grid, smem, bytes, flops, st);
    default: return launch<false, IT_EXPERT_OUT_F32>(ma, mw, p, grid, smem, bytes, flops, st);
  }
}
