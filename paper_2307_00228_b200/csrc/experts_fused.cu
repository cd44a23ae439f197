// Both products of an expert in one kernel, for rows that fit an SM: a tile of 128 places keeps its input in shared memory and its result
// in TMEM while the hidden columns go by, 128 at a time, so that the hidden row is neither written to nor read from device memory:
//   S = X W1[:, chunk]  (TMEM)  ->  P = bf16( act( S + b1 ) )  (TMEM, where S lay)  ->  O += P W2[chunk, :]  (TMEM)
// Gated: a chunk is 64 columns of the gate and the 64 that it gates.  With the hidden row in memory the two products of 1M vertices, 2 of 16,
// 128-512-128, moved 6 GB, 4 of them hidden rows, and took 1160 us at 5.2 TB/s.
//
// Warps: 0 and 1 fetch W1 and W2 (TMA), 2 and 3 issue the MMAs of S and of O, 4-11 make P, 12-15 fetch the rows of X by place (16-byte asynchronous
// copies) and store O: sixteen, which leave 128 registers a thread.  Nearly every one of these was the slowest once: one issuing warp for S and O with
// a stage of weights per k-block 3300 cycles a chunk (a wait costs it some 160, a commit 95), one warp for the rows 2500 (100 a copy), one
// producer for both weights 570 of waiting for W2 behind W1, rows fetched by the warps that make P 400.
// S and P are buffered twice, O twice where it has at most 128 columns.
// Waits are bounded as in the other products.
#include <type_traits>

#include "experts_tc.cuh"

namespace {

constexpr int FU_W1_WARP = 0, FU_W2_WARP = 1, FU_S_WARP = 2, FU_MMA_WARP = 3 /* of O */, FU_P_WARP0 = 4, FU_P_WARPS = 8, FU_O_WARP0 = 12, FU_O_WARPS = 4;
constexpr int FU_THREADS = 32 * (FU_O_WARP0 + FU_O_WARPS);
constexpr int FU_XBLOCK = TC_BM * TC_KBLOCK_BYTES;
constexpr int FU_MAX_STAGES = 4;     // of either ring of weights
constexpr int FU_BACKOFF = 32;       // ns between polls
constexpr int FU_S_COLS = 128;       // accumulator columns of a chunk

struct FuParams {
  const int32_t *order, *tile_expert, *n_tiles;
  const void *x;
  const float *x_scale, *w_scale, *b1, *b2, *weights;
  int tiles_max, top_k, n_experts;
  int in_bytes, kbx;                 // bytes of a row of X, its k-blocks
  int hidden, n1, chunks, chunk_hidden;   // columns of W1; chunks of 128 (gated: 64) hidden columns
  int out, bn;                       // columns of the result, and padded to panels
  int kb1, stages1, stage1;          // W1: k-blocks of a stage, stages, bytes of one
  int kb2, stages2, stage2;          // W2: of 64 hidden columns each
  int x_slots, o_bufs;
  int act;
  void *dst;
  int *status;
  uint32_t spin_limit;
  int no_loads;
};

template <bool EIGHT, bool GATED, bool DIRECT>
__global__ void __launch_bounds__(FU_THREADS, 1)
expert_fused_kernel(const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ CUtensorMap map_w2, const FuParams p) {
  extern __shared__ __align__(1024) unsigned char base[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int BK1 = EIGHT ? 128 : 64;              // elements of a k-block of X, and columns of a panel of W1
  constexpr int STAGING = 4096;                      // per storing warp: 32 rows of 128 bytes
  unsigned char *x_s = base;
  unsigned char *w1_s = x_s + (size_t)p.x_slots * p.kbx * FU_XBLOCK;
  unsigned char *w2_s = w1_s + (size_t)p.stages1 * p.stage1;
  unsigned char *staging = w2_s + (size_t)p.stages2 * p.stage2;
  float *p_consts = reinterpret_cast<float *>(staging + FU_O_WARPS * STAGING);   // [8 warps][2][64 bias | 64 scale]
  float *o_consts = p_consts + FU_P_WARPS * 2 * (EIGHT ? 128 : 64);               // [4 warps][256] b2
  int32_t *o_place = reinterpret_cast<int32_t *>(o_consts + FU_O_WARPS * 256);    // [128]
  uint64_t *w1_full = reinterpret_cast<uint64_t *>(o_place + TC_BM);
  uint64_t *w1_empty = w1_full + FU_MAX_STAGES;
  uint64_t *w2_full = w1_empty + FU_MAX_STAGES;
  uint64_t *w2_empty = w2_full + FU_MAX_STAGES;
  uint64_t *x_full = w2_empty + FU_MAX_STAGES;   // [2]
  uint64_t *x_empty = x_full + 2;               // [2]
  uint64_t *s_full = x_empty + 2;               // [2]
  uint64_t *s_free = s_full + 2;                // [2]  the product that read P from this buffer is over
  uint64_t *p_full = s_free + 2;                // [2]
  uint64_t *o_full = p_full + 2;                // [2]
  uint64_t *o_empty = o_full + 2;               // [2]
  uint64_t *mma_done = o_empty + 2;             // [2]  every MMA of S, of O is over
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 2);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < FU_MAX_STAGES; ++s) {
      mbar_init(&w1_full[s], 1);
      mbar_init(&w1_empty[s], 1);
      mbar_init(&w2_full[s], 1);
      mbar_init(&w2_empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&x_full[a], 32 * FU_O_WARPS);
      mbar_init(&x_empty[a], 1);
      mbar_init(&s_free[a], 1);
      mbar_init(&mma_done[a], 1);
      mbar_init(&s_full[a], 1);
      mbar_init(&p_full[a], FU_P_WARPS);
      mbar_init(&o_full[a], 1);
      mbar_init(&o_empty[a], FU_O_WARPS);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == FU_MMA_WARP) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  it_allow_next();
  it_wait_prior();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot, s_col = (uint32_t)(p.o_bufs * p.bn);   // O first, then the two S
  int m_tiles = *p.n_tiles;
  m_tiles = m_tiles < p.tiles_max ? m_tiles : p.tiles_max;

  if (warp == FU_W1_WARP || warp == FU_W2_WARP) {
    // ------------------------------------------------------------------ weights: one of the two, a ring each
    const bool first = warp == FU_W1_WARP;
    uint64_t *full = first ? w1_full : w2_full, *empty = first ? w1_empty : w2_empty;
    const uint32_t stages = (uint32_t)(first ? p.stages1 : p.stages2), stage_bytes = (uint32_t)(first ? p.stage1 : p.stage2);
    unsigned char *ring = first ? w1_s : w2_s;
    const int kbs = first ? p.kbx : p.chunk_hidden / 64, per_stage = first ? p.kb1 : p.kb2;   // k-blocks of a chunk, of a stage
    const int panels = first ? 128 / BK1 : p.bn / 64, block_bytes = first ? FU_XBLOCK : p.bn * TC_KBLOCK_BYTES, panel_bytes = block_bytes / panels;
    const int kb_lane = lane / panels, panel = lane % panels;
    uint32_t stage = 0, phase = 0;
    bool ok = !p.no_loads, came_round = false;
    int e_next = (int)blockIdx.x < m_tiles ? p.tile_expert[blockIdx.x] : 0;
    for (int m = blockIdx.x; m < m_tiles && ok; m += gridDim.x) {
      const int e = e_next;
      if (m + (int)gridDim.x < m_tiles) e_next = p.tile_expert[m + gridDim.x];
      for (int c = 0; c < p.chunks && ok; ++c)
        for (int kb0 = 0; kb0 < kbs; kb0 += per_stage) {
          const int n = kbs - kb0 < per_stage ? kbs - kb0 : per_stage;
          if (lane == 0) {
            ok = mbar_wait(&empty[stage], phase ^ 1u, abort_flag, p.spin_limit, FU_BACKOFF);
            if (ok) mbar_arrive_expect_tx(&full[stage], (uint32_t)(n * block_bytes));
          }
          ok = __shfl_sync(0xffffffffu, (int)ok, 0);
          if (!ok) break;
          if (kb_lane < n) {
            unsigned char *to = ring + (size_t)stage * stage_bytes + lane * panel_bytes;
            if (first) tma_load_3d(to, &map_w1, GATED ? panel * p.hidden + c * 64 : c * 128 + panel * BK1, (kb0 + kb_lane) * BK1, e, &full[stage]);
            else tma_load_3d(to, &map_w2, panel * 64, c * p.chunk_hidden + (kb0 + kb_lane) * 64, e, &full[stage]);
          }
          __syncwarp();
          if (++stage == stages) { stage = 0; phase ^= 1u; came_round = true; }
        }
    }
    __syncwarp();
    if (lane == 0) ring_drain(full, stages, stage, phase, came_round);
  } else if (warp == FU_S_WARP) {
    // ------------------------------------------------------------------ S = X W1: chunk number g of this CTA into buffer g % 2
    const uint32_t fmt = EIGHT ? 0u : 1u, lead = lane == 0;
    const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | (1u << 16) | ((uint32_t)(FU_S_COLS >> 3) << 17) | ((uint32_t)(TC_BM >> 4) << 24);
    uint32_t stage = 0, phase = 0, slot = 0, x_phase = 0, g = 0;
    bool ok = true;
    for (int m = blockIdx.x; m < m_tiles && ok; m += gridDim.x) {
      ok = ex_wait_warp(&x_full[slot], x_phase, abort_flag, p.spin_limit);
      if (!ok) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the rows were written by other threads' copies
      const uint64_t x_d = make_desc(smem_u32(x_s) + slot * (uint32_t)(p.kbx * FU_XBLOCK));
      for (int c = 0; c < p.chunks && ok; ++c, ++g) {
        const uint32_t d = tmem_base + s_col + (g & 1u) * FU_S_COLS;
        for (int kb0 = 0; kb0 < p.kbx && ok; kb0 += p.kb1) {
          ok = ex_wait_warp(&w1_full[stage], phase, abort_flag, p.spin_limit);
          // the chunk before the last one's P lies where this S goes (waited for last: the weights are long there, and a wait takes its time)
          if (ok && kb0 == 0 && g >= 2) ok = ex_wait_warp(&s_free[g & 1u], ((g >> 1) & 1u) ^ 1u, abort_flag, p.spin_limit);
          if (!ok) break;
          tc_fence_after();   // other warps wrote that P and read it in an MMA: what is issued here stays behind them
          const uint64_t b_d = make_desc_mn(smem_u32(w1_s) + stage * (uint32_t)p.stage1, BK1 * TC_KBLOCK_BYTES);
          for (int i = 0; i < p.kb1 && kb0 + i < p.kbx; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              ex_mma<EIGHT>(lead, d, x_d + (kb0 + i) * (FU_XBLOCK / 16) + k * 2, b_d + i * (FU_XBLOCK / 16) + k * (BK1 * TC_KBLOCK_BYTES / 64), idesc, (kb0 | i | k) != 0);
          }
          ex_commit(lead, &w1_empty[stage]);
          if (++stage == (uint32_t)p.stages1) { stage = 0; phase ^= 1u; }
        }
        if (ok) ex_commit(lead, &s_full[g & 1u]);
      }
      if (ok) ex_commit(lead, &x_empty[slot]);
      if (++slot == (uint32_t)p.x_slots) { slot = 0; x_phase ^= 1u; }
    }
    ex_commit(lead, &mma_done[0]);
    mbar_drain(&mma_done[0], 0);
  } else if (warp == FU_MMA_WARP) {
    // ------------------------------------------------------------------ O += P W2: tile number t of this CTA into buffer t % o_bufs
    const uint32_t lead = lane == 0;
    const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(p.bn >> 3) << 17) | ((uint32_t)(TC_BM >> 4) << 24);
    uint32_t stage = 0, phase = 0, g = 0, t = 0;
    bool ok = true;
    for (int m = blockIdx.x; m < m_tiles && ok; m += gridDim.x, ++t) {
      const uint32_t ob = p.o_bufs == 2 ? t & 1u : 0u, ot = p.o_bufs == 2 ? t >> 1 : t, d = tmem_base + ob * (uint32_t)p.bn;
      ok = ex_wait_warp(&o_empty[ob], (ot & 1u) ^ 1u, abort_flag, p.spin_limit);
      for (int c = 0; c < p.chunks && ok; ++c, ++g) {
        const uint32_t pt = tmem_base + s_col + (g & 1u) * FU_S_COLS;
        for (int kb0 = 0; kb0 < p.chunk_hidden / 64 && ok; kb0 += p.kb2) {
          ok = ex_wait_warp(&w2_full[stage], phase, abort_flag, p.spin_limit);
          if (ok && kb0 == 0) ok = ex_wait_warp(&p_full[g & 1u], (g >> 1) & 1u, abort_flag, p.spin_limit);
          if (!ok) break;
          tc_fence_after();
          const uint64_t b_d = make_desc_mn(smem_u32(w2_s) + stage * (uint32_t)p.stage2, 8192);
          for (int i = 0; i < p.kb2; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k)   // where the warps that make P leave it: 32 columns of theirs hold 64 hidden columns, gated 16 hold 32
              ex_mma_tmem_a(lead, d, GATED ? pt + (k >> 1) * 32 + (k & 1) * 8 : pt + (kb0 + i) * 64 + k * 8, b_d + i * (p.bn * 8) + k * 128, idesc,
                            (c | kb0 | i | k) != 0);
          }
          ex_commit(lead, &w2_empty[stage]);
          if (++stage == (uint32_t)p.stages2) { stage = 0; phase ^= 1u; }
        }
        if (ok) ex_commit(lead, &s_free[g & 1u]);
      }
      if (ok) ex_commit(lead, &o_full[ob]);
    }
    ex_commit(lead, &mma_done[1]);
    mbar_drain(&mma_done[1], 0);
  } else if (warp < FU_P_WARP0 + FU_P_WARPS) {
    // ------------------------------------------------------------------ P: a thread per row, 64 accumulator columns a warp (gated: 32 of the gate, 32 gated)
    const int quarter = warp & 3, sub = (warp - FU_P_WARP0) >> 2;   // a warp may only touch TMEM lanes [32 * (warp % 4), +32)
    float *consts = p_consts + (warp - FU_P_WARP0) * 2 * (EIGHT ? 128 : 64);
    // two constants a lane, those of the columns 2 lane and 2 lane + 1 (gated: of column lane of either half), fetched a chunk ahead
    struct Two { float2 b, s; };
    auto fetch = [&](int e, int c) {
      Two q{make_float2(0.f, 0.f), make_float2(1.f, 1.f)};
      const int64_t row = (int64_t)e * p.n1;
      if constexpr (GATED) {
        const int h = c * 64 + sub * 32 + lane;
        if (h < p.hidden && p.b1) q.b = make_float2(p.b1[row + h], p.b1[row + p.hidden + h]);
      } else {
        const int h = c * 128 + sub * 64 + lane * 2;
        if (h < p.hidden) {   // (hidden is a multiple of 8)
          if (p.b1) q.b = *reinterpret_cast<const float2 *>(p.b1 + row + h);
          if constexpr (EIGHT) q.s = *reinterpret_cast<const float2 *>(p.w_scale + row + h);
        }
      }
      return q;
    };
    const uint32_t floor2 = p.act == IT_ACT_RELU ? 0u : 0xff80ff80u;
    uint32_t g = 0;
    bool ok = true;
    int e_next = (int)blockIdx.x < m_tiles ? p.tile_expert[blockIdx.x] : 0;
    int place_next = EIGHT && (int)blockIdx.x < m_tiles ? p.order[(int64_t)blockIdx.x * TC_BM + quarter * 32 + lane] : -1;
    float xs_next = EIGHT && place_next >= 0 ? p.x_scale[place_next / p.top_k] : 1.f;
    Two next{};
    if ((int)blockIdx.x < m_tiles) next = fetch(e_next, 0);
    for (int m = blockIdx.x; m < m_tiles && ok; m += gridDim.x) {
      const int e = e_next, after = m + gridDim.x;
      const uint32_t xw = __float_as_uint(xs_next);
      const uint64_t xs2 = pack2(xw, xw);
      if (after < m_tiles) {
        e_next = p.tile_expert[after];
        if constexpr (EIGHT) place_next = p.order[(int64_t)after * TC_BM + quarter * 32 + lane];
      }
      for (int c = 0; c < p.chunks; ++c, ++g) {
        float *k = consts + (g & 1u) * (EIGHT ? 128 : 64);
        __syncwarp();
        if constexpr (GATED) { k[lane] = next.b.x; k[32 + lane] = next.b.y; }
        else {
          *reinterpret_cast<float2 *>(k + 2 * lane) = next.b;
          if constexpr (EIGHT) *reinterpret_cast<float2 *>(k + 64 + 2 * lane) = next.s;
        }
        __syncwarp();
        if (c + 1 < p.chunks) next = fetch(e, c + 1);
        else if (after < m_tiles) {
          next = fetch(e_next, 0);
          if constexpr (EIGHT) xs_next = place_next >= 0 ? p.x_scale[place_next / p.top_k] : 1.f;
        }
        ok = mbar_wait(&s_full[g & 1u], (g >> 1) & 1u, abort_flag, p.spin_limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t st = tmem_base + ((uint32_t)(quarter * 32) << 16) + s_col + (g & 1u) * FU_S_COLS;
        // 32 columns of S, scaled, with their bias
        auto scaled = [&](const uint32_t (&r)[32], int at, uint64_t (&v)[16]) {
          const ulonglong2 *b = reinterpret_cast<const ulonglong2 *>(k + at);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const ulonglong2 bb = b[i];
            uint64_t lo = pack2(r[4 * i], r[4 * i + 1]), hi = pack2(r[4 * i + 2], r[4 * i + 3]);
            if constexpr (EIGHT) {
              const ulonglong2 f = reinterpret_cast<const ulonglong2 *>(k + 64 + at)[i];
              lo = fma2(mul2(lo, xs2), f.x, bb.x);
              hi = fma2(mul2(hi, xs2), f.y, bb.y);
            } else {
              lo = add2(lo, bb.x);
              hi = add2(hi, bb.y);
            }
            v[2 * i] = lo;
            v[2 * i + 1] = hi;
          }
        };
        // left: hidden columns from the first of these 32 on.  What lies behind the last one is 0: zeros for W1 times an infinite state would be NaN, and stay so
        // times zeros for W2
        auto pack = [&](const uint64_t (&v)[16], uint32_t (&w)[16], bool cut, int left) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 f = unpack2(v[i]);
            w[i] = bf16x2_of(f.x, f.y);
            if (cut) w[i] = max_bf16x2(w[i], floor2);
          }
          if (left < 32) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (2 * i >= left) w[i] = 0u;
          }
        };
        if constexpr (GATED) {
          uint32_t r[32], u[32], w[16];
          tmem_ld32(st + (uint32_t)(sub * 32), r);
          tmem_ld32(st + 64u + (uint32_t)(sub * 32), u);
          tmem_ld_wait();
          uint64_t v[16], q[16];
          scaled(r, 0, v);
          expert_act(v, p.act);
          scaled(u, 32, q);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = mul2(v[i], q[i]);
          pack(v, w, false, 32);   // (gated, an infinite state has no finite row: 0 times what is gated is NaN)
          tmem_st16(st + (uint32_t)(sub * 32), w);
        } else {
          // (P of the first 32 columns takes the place of 16 of them, which have been read)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32], w[16];
            uint64_t v[16];
            tmem_ld32(st + (uint32_t)(sub * 64 + h * 32), r);
            tmem_ld_wait();
            scaled(r, h * 32, v);
            if (p.act != IT_ACT_RELU) expert_act(v, p.act);
            pack(v, w, true, p.hidden - c * 128 - sub * 64 - h * 32);
            tmem_st16(st + (uint32_t)(sub * 64 + h * 16), w);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[g & 1u]);
      }
    }
  } else {
    // ------------------------------------------------------------------ rows of X, by place; and O: rows of the result, through a staging tile
    const int quarter = warp & 3;
    constexpr int ESIZE = DIRECT ? 2 : 4, ROW = 128;
    const uint32_t stage_s = smem_u32(staging) + (uint32_t)(warp - FU_O_WARP0) * STAGING;
    const int row0 = lane >> 3, piece = lane & 7;
    const uint32_t put = stage_s + (uint32_t)lane * ROW + (uint32_t)((lane & 7) << 4);
    const uint32_t row4 = 4u * (uint32_t)p.out * ESIZE;
    float *bias = o_consts + (warp - FU_O_WARP0) * 256;
    int32_t *places = o_place + quarter * 32;
    // 32 rows of tile number t into slot t % x_slots.  Two slots: tile t + 2 once O of tile t is there, whose rows are read then; one: tile t + 1
    // once the last S of tile t is.
    int x_place = -1;   // of the rows that are fetched next
    auto look_x = [&](int m) {
      if (m < m_tiles) x_place = p.order[(int64_t)m * TC_BM + quarter * 32 + lane];
    };
    auto fetch_x = [&](uint32_t slot) {
      const int row = x_place < 0 ? -1 : x_place / p.top_k;
      const uint32_t to = smem_u32(x_s) + slot * (uint32_t)(p.kbx * FU_XBLOCK) + (uint32_t)(quarter * 32 + row0) * TC_KBLOCK_BYTES;
      const uint32_t even = to + (uint32_t)((piece ^ row0) << 4), odd = to + (uint32_t)((piece ^ (4 + row0)) << 4);
      const unsigned char *src[8];
      uint32_t bytes[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = __shfl_sync(0xffffffffu, row, i * 4 + row0);
        src[i] = reinterpret_cast<const unsigned char *>(p.x) + (int64_t)(r < 0 ? 0 : r) * p.in_bytes + piece * 16;
        bytes[i] = r < 0 ? 0u : 16u;
      }
      for (int kb = 0; kb < p.kbx; ++kb) {
        const bool in = kb * TC_KBLOCK_BYTES + piece * 16 < p.in_bytes;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          cp_async16(((i & 1) ? odd : even) + (uint32_t)(i * 512) + (uint32_t)kb * FU_XBLOCK, in ? src[i] + kb * TC_KBLOCK_BYTES : src[i] - piece * 16, in ? bytes[i] : 0u);
      }
      cp_async_arrive(&x_full[slot]);
    };
    const int stride = (int)gridDim.x, ahead = p.x_slots;   // tiles that the rows are ahead
    for (int i = 0; i < ahead; ++i)
      if ((int64_t)blockIdx.x + (int64_t)i * stride < m_tiles && !p.no_loads) {
        look_x(blockIdx.x + i * stride);
        fetch_x((uint32_t)i);
      }
    uint32_t t = 0, x_slot = 0, x_phase = 0;
    for (int m = blockIdx.x; m < m_tiles; m += stride, ++t) {
      const int64_t pos0 = (int64_t)m * TC_BM + quarter * 32;
      const int place = p.order[pos0 + lane], e = p.tile_expert[m];
      const bool more = (int64_t)m + (int64_t)ahead * stride < m_tiles;
      if (more) look_x(m + ahead * stride);
      const float weight = DIRECT && place >= 0 ? p.weights[place] : 1.f;
      const uint64_t weight2 = pack2(__float_as_uint(weight), __float_as_uint(weight));
      __syncwarp();
      places[lane] = place;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = i * 128 + lane * 4;
        *reinterpret_cast<float4 *>(bias + c) = p.b2 && c < p.out ? *reinterpret_cast<const float4 *>(p.b2 + (int64_t)e * p.out + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      __syncwarp();
      const uint32_t ob = p.o_bufs == 2 ? t & 1u : 0u, ot = p.o_bufs == 2 ? t >> 1 : t;
      bool ok = true;
      if (ahead == 2) ok = mbar_wait(&o_full[ob], ot & 1u, abort_flag, p.spin_limit, 4 * FU_BACKOFF);
      if (ok && more) ok = mbar_wait(&x_empty[x_slot], x_phase, abort_flag, p.spin_limit, FU_BACKOFF);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (more) fetch_x(x_slot);
      if (++x_slot == (uint32_t)p.x_slots) { x_slot = 0; x_phase ^= 1u; }
      if (ahead != 2) ok = mbar_wait(&o_full[ob], ot & 1u, abort_flag, p.spin_limit, 4 * FU_BACKOFF);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + ob * (uint32_t)p.bn;
      unsigned char *to = reinterpret_cast<unsigned char *>(p.dst) + (DIRECT ? 0 : (pos0 + row0) * p.out) * ESIZE + piece * 16;
      const unsigned real = __ballot_sync(0xffffffffu, place >= 0) >> row0;   // bit 4 i: whether the i-th row that this lane stores parts of is one
      auto flush = [&](int c, bool both) {   // the staged pieces of rows, from column c on
        __syncwarp();
        const bool in = c + piece * (16 / ESIZE) < p.out && (both || piece < 4);
        const uint32_t even = stage_s + (uint32_t)row0 * ROW + (uint32_t)((piece ^ row0) << 4), odd = stage_s + (uint32_t)row0 * ROW + (uint32_t)((piece ^ (4 + row0)) << 4);
        uint4 d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(d[i].x), "=r"(d[i].y), "=r"(d[i].z), "=r"(d[i].w) : "r"(((i & 1) ? odd : even) + 512u * i) : "memory");
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (in && ((real >> (4 * i)) & 1u)) *reinterpret_cast<uint4 *>(to + (DIRECT ? (int64_t)places[4 * i + row0] * p.out * ESIZE : (int64_t)((uint64_t)i * row4)) + c * ESIZE) = d[i];
        __syncwarp();
      };
      for (int c = 0; c < p.out; c += 32) {
        uint32_t r[32];
        tmem_ld32(taddr + (uint32_t)c, r);
        tmem_ld_wait();
        const ulonglong2 *b = reinterpret_cast<const ulonglong2 *>(bias + c);
        uint64_t v[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const ulonglong2 bb = b[i];
          v[2 * i] = add2(pack2(r[4 * i], r[4 * i + 1]), bb.x);
          v[2 * i + 1] = add2(pack2(r[4 * i + 2], r[4 * i + 3]), bb.y);
        }
        if constexpr (DIRECT) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 f = unpack2(mul2(v[i], weight2));
            w[i] = bf16x2_of(f.x, f.y);
          }
          const int half = (c >> 5) & 1;
#pragma unroll
          for (int i = 0; i < 4; ++i) st_shared_v4(put ^ (16u * (4 * half + i)), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          if (half == 1 || c + 32 >= p.out) flush(c - 32 * half, half == 1);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 f0 = unpack2(v[2 * i]), f1 = unpack2(v[2 * i + 1]);
            st_shared_v4(put ^ (16u * i), __float_as_uint(f0.x), __float_as_uint(f0.y), __float_as_uint(f1.x), __float_as_uint(f1.y));
          }
          flush(c, true);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&o_empty[ob]);
    }
    __syncwarp();
    cp_async_wait_all();
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.status, 1);
  if (warp == FU_MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <bool EIGHT, bool GATED, bool DIRECT>
it_status launch(const CUtensorMap &m1, const CUtensorMap &m2, const FuParams &p, int grid, int smem, double bytes, double flops, cudaStream_t st) {
  IT_CUDA_TRY(cudaFuncSetAttribute(expert_fused_kernel<EIGHT, GATED, DIRECT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  IT_LAUNCH(IT_K_EXPERT_GEMM, bytes, flops, st,
            IT_CUDA_TRY((it_launch_pdl(expert_fused_kernel<EIGHT, GATED, DIRECT>, dim3((unsigned)grid), dim3(FU_THREADS), smem, st, m1, m2, p))));
  return IT_OK;
}

}  // namespace

// Rows of X of up to 512 bytes (a tile of them fits shared memory twice beside the weights' stages), results of up to 256 columns (that
// fit TMEM beside the two chunks); not gated in 8 bits, whose panels of 128 columns do not divide into gate and gated.
bool it_experts_fused(const it_experts_desc &d) {
  const int in_bytes = d.in_dim * (d.in_dtype == IT_E4M3 ? 1 : 2);
  return d.hidden_dim > 0 && d.feat_dtype == IT_BF16 && in_bytes <= 512 && d.out_dim <= 256 && !(d.gated && d.in_dtype == IT_E4M3);
}

it_status it_launch_experts_fused(const it_experts_args &a, const it_experts_plan &q, void *dst, uint32_t spin_limit, int no_loads, cudaStream_t st) {
  const it_experts_desc &d = a.d;
  const bool eight = d.in_dtype == IT_E4M3, gated = d.gated != 0, direct = d.top_k == 1;
  const int elem = eight ? 1 : 2, BK = TC_KBLOCK_BYTES / elem;
  FuParams p{};
  p.order = q.order; p.tile_expert = q.tile_expert; p.n_tiles = q.n_tiles; p.tiles_max = (int)q.tiles_max;
  p.x = a.x; p.x_scale = a.x_scale; p.w_scale = d.w1_scale; p.b1 = d.b1; p.b2 = d.b2; p.weights = a.weights;
  p.top_k = d.top_k; p.n_experts = d.n_experts; p.in_bytes = d.in_dim * elem; p.kbx = (d.in_dim + BK - 1) / BK;
  p.hidden = d.hidden_dim; p.n1 = a.n1; p.chunk_hidden = gated ? 64 : 128; p.chunks = (d.hidden_dim + p.chunk_hidden - 1) / p.chunk_hidden;
  p.out = d.out_dim; p.bn = (d.out_dim + 63) / 64 * 64; p.o_bufs = p.bn <= 128 ? 2 : 1;
  p.act = d.act; p.dst = dst; p.status = a.status; p.spin_limit = spin_limit ? spin_limit : TC_SPIN_LIMIT; p.no_loads = no_loads;

  const cuuint64_t d1[3] = {(cuuint64_t)a.n1, (cuuint64_t)d.in_dim, (cuuint64_t)d.n_experts}, s1[2] = {(cuuint64_t)a.n1 * elem, (cuuint64_t)a.n1 * elem * (cuuint64_t)d.in_dim};
  const cuuint64_t d2[3] = {(cuuint64_t)d.out_dim, (cuuint64_t)d.hidden_dim, (cuuint64_t)d.n_experts}, s2[2] = {(cuuint64_t)d.out_dim * 2, (cuuint64_t)d.out_dim * 2 * (cuuint64_t)d.hidden_dim};
  const cuuint32_t b1[3] = {(cuuint32_t)BK, (cuuint32_t)BK, 1}, b2[3] = {64, 64, 1};
  CUtensorMap m1, m2;
  IT_TRY(encode(&m1, eight, d.W1, 3, d1, s1, b1));
  IT_TRY(encode(&m2, false, d.W2, 3, d2, s2, b2));

  const int fixed = FU_O_WARPS * 4096 + FU_P_WARPS * 2 * (eight ? 128 : 64) * 4 + FU_O_WARPS * 256 * 4 + TC_BM * 4 + (4 * FU_MAX_STAGES + 17) * 8;
  // a stage of weights: two k-blocks (W2: of up to 128 columns), or the one there is
  p.kb1 = p.kbx < 2 ? 1 : 2; p.stage1 = p.kb1 * FU_XBLOCK;
  p.kb2 = gated || p.bn > 128 ? 1 : 2; p.stage2 = p.kb2 * p.bn * TC_KBLOCK_BYTES;
  p.x_slots = p.kbx <= 2 ? 2 : 1;
  const int room = (227 * 1024 - fixed - p.x_slots * p.kbx * FU_XBLOCK) / (p.stage1 + p.stage2);
  p.stages1 = p.stages2 = room < FU_MAX_STAGES ? room : FU_MAX_STAGES;
  const int smem = fixed + p.x_slots * p.kbx * FU_XBLOCK + p.stages1 * p.stage1 + p.stages2 * p.stage2;
  const int grid = (int)(q.tiles_max < a.sms ? q.tiles_max : a.sms);
  const double places = (double)a.n * d.top_k;
  const double flops = 2.0 * places * ((double)d.in_dim * a.n1 + (double)d.hidden_dim * d.out_dim), bytes = places * (p.in_bytes + (double)d.out_dim * (direct ? 2 : 4));
#define IT_FU_LAUNCH(EIGHT, GATED, DIRECT) return launch<EIGHT, GATED, DIRECT>(m1, m2, p, grid, smem, bytes, flops, st)
  if (eight) { if (direct) IT_FU_LAUNCH(true, false, true); else IT_FU_LAUNCH(true, false, false); }
  if (gated) { if (direct) IT_FU_LAUNCH(false, true, true); else IT_FU_LAUNCH(false, true, false); }
  if (direct) IT_FU_LAUNCH(false, false, true);
  IT_FU_LAUNCH(false, false, false);
#undef IT_FU_LAUNCH
}
