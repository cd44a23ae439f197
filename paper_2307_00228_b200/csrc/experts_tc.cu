// The products of it_experts_forward on the tensor cores: one persistent, warp-specialised kernel over tiles of 128 places of one expert,
//   D[128, cols] = A[places, K] * W[expert][K, cols]
// with tcgen05.mma (accumulators in TMEM, two of them, so that a tile's epilogue runs beside the next tile's products), operands
// staged in 128-byte-swizzled k-blocks.  The rows of A are fetched where they lie, by the place's vertex, with 16-byte asynchronous copies of four
// warps (TMA gathers of four rows took 52 cycles each, 1650 a k-block: 40k vertices, 4 of 32, 768-1024 gated 730 us); rows in order and the
// weights come by TMA, the weights taken as they are, [K, columns], which makes B an MN-major operand, so nothing is transposed or prepared.
// bf16 (kind::f16), e4m3 (kind::f8f6f4), and fp32 as three bf16 parts a value in six products per k-block, the smallest first
// (what is left out is 2^-24 of a term).
//
// Every wait on an mbarrier is bounded: when one gives up, the CTA raises a flag that all roles poll, waits for its copies and products in
// flight, frees its TMEM and returns, and a status word in global memory is set.
#include <type_traits>

#include "experts_tc.cuh"

namespace {

constexpr int EX_FETCH_WARPS = 4;  // rows found by place: each fetches a quarter of a tile's rows; the weights and rows in order: the first, by TMA
constexpr int EX_MMA_WARP = 4, EX_META_WARP = 5, EX_EPI_WARP0 = 6;
constexpr int EX_EPI_WARPS = 8;    // two per TMEM lane quarter, each takes every other 64 bytes of a row
constexpr int EX_EPI_SUBS = EX_EPI_WARPS / 4;
constexpr int EX_THREADS = 32 * (EX_EPI_WARP0 + EX_EPI_WARPS);
constexpr int EX_STAGE_A = TC_BM * TC_KBLOCK_BYTES;
// Per epilogue warp: 32 rows of 64 bytes; rows of the output that lie apart are written 128 bytes at a time (at the cost of a stage of operands):
// 1.5M rows of 512 bytes in halves of a line 339 us, by two warps in turn 634.
__host__ __device__ constexpr bool ex_direct(it_expert_store s) { return s == IT_EXPERT_OUT_BF16 || s == IT_EXPERT_OUT_F32; }
__host__ __device__ constexpr int ex_staging(it_expert_store s) { return ex_direct(s) ? 4096 : 2048; }
// What the epilogue of a tile needs besides the product: places of the rows, their weights and scales, bias and scale of the columns.
struct ExMeta { int32_t place[TC_BM]; float weight[TC_BM]; float bias[256]; };
struct ExMetaEight : ExMeta { float xs[TC_BM]; float scale[256]; };
constexpr int EX_MAX_STAGES = 8;
constexpr int EX_SLICE = 4;        // k-blocks of a slice (LONG_SUMS)
constexpr int EX_EPI_BACKOFF = 64, EX_TMA_BACKOFF = 32;   // ns between polls

struct ExParams {
  const int32_t *order, *tile_expert, *n_tiles;
  const void *A;
  int tiles_max;
  int n_splits, bn, cols_per_tile;   // column tiles; columns of an accumulator; columns of the result in a tile (gated: bn / 2)
  int K, kb;                         // k-blocks
  int stages;
  int box_panels;                    // panels of W that one copy fetches, or 0: a copy each
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

// the parts of A and W that pass i of the six multiplies, smallest products first
__device__ __forceinline__ void pass_parts(int i, int *pa, int *pb) {
  constexpr uint32_t A = 0x001102u, B = 0x010120u;   // nibble i: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
  *pa = (int)((A >> (4 * i)) & 15u);
  *pb = (int)((B >> (4 * i)) & 15u);
}

// TRI (fp32, K up to 256): a stage holds the three parts of a k-block of either operand, and an accumulator of its own takes the small products.
// LONG_SUMS (fp32, K above 256): slice by slice of K, each with all its six products; the epilogue adds the slices up, rounding to nearest, in the second
// accumulator's place.
enum ExForm { EX_PLAIN, EX_TRI, EX_LONG_SUMS };
template <bool EIGHT, it_expert_store STORE, bool GATED, ExForm FORM>
__global__ void __launch_bounds__(EX_THREADS, 1)
expert_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const ExParams p) {
  extern __shared__ __align__(1024) unsigned char base[];   // (the swizzle goes by addresses: stages start at multiples of 1024)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int BK = EIGHT ? 128 : 64;                  // elements of a k-block, and columns of a panel
  constexpr int PANEL = BK * TC_KBLOCK_BYTES;           // bytes of a panel of W: BK rows x 128 bytes
  constexpr bool TRI = FORM == EX_TRI, LONG_SUMS = FORM == EX_LONG_SUMS;
  constexpr int P = TRI ? 3 : 1;                        // parts in a stage: of A, then of W
  const int b_bytes = p.bn * TC_KBLOCK_BYTES, stage_bytes = P * (EX_STAGE_A + b_bytes);

  unsigned char *staging = base + (size_t)p.stages * stage_bytes;
  using Meta = std::conditional_t<EIGHT, ExMetaEight, ExMeta>;
  Meta *meta = reinterpret_cast<Meta *>(staging + EX_EPI_WARPS * ex_staging(STORE));   // [2], one per accumulator
  uint64_t *full = reinterpret_cast<uint64_t *>(meta + 2);   // [stages]
  uint64_t *empty = full + EX_MAX_STAGES;      // [stages]
  uint64_t *acc_full = empty + EX_MAX_STAGES;  // [2]
  uint64_t *acc_empty = acc_full + 2;          // [2]
  uint64_t *meta_full = acc_empty + 2;         // [2]
  uint64_t *mma_done = meta_full + 2;          // [1]
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 1);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  uint32_t tmem_cols = 32;
  while (tmem_cols < (TRI ? 4u : 2u) * (uint32_t)p.bn) tmem_cols <<= 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], p.gather_div ? 32 * EX_FETCH_WARPS + 1 : 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&acc_full[a], 1);
      mbar_init(&meta_full[a], 1);
      mbar_init(&acc_empty[a], EX_EPI_WARPS);
    }
    mbar_init(mma_done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == EX_MMA_WARP) {
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
  const uint32_t splits = (uint32_t)p.n_splits, n_tiles = (uint32_t)m_tiles * splits;   // (below 2^31)
  constexpr int PASSES = LONG_SUMS ? 6 : 1;   // walks over the k-blocks
  const int slices = LONG_SUMS ? (p.kb + EX_SLICE - 1) / EX_SLICE : 1;
  constexpr uint32_t bufs = LONG_SUMS ? 1u : 2u;
  const uint32_t acc_stride = (uint32_t)p.bn * (TRI ? 2u : 1u);   // accumulators of tiles in flight

  if (warp < EX_FETCH_WARPS) {
    // ------------------------------------------------------------------ producers: rows found by place by all four warps, 16 bytes a lane;
    // weights, and rows in order, by TMA from the first
    uint32_t stage = 0, phase = 0;
    const bool gather = !TRI && p.gather_div > 0;
    bool ok = !p.no_loads && (warp == 0 || gather), came_round = false;
    const uint32_t tma_bytes = P * ((gather ? 0 : EX_STAGE_A) + b_bytes);
    const int chunk = lane & 7;
    uint32_t dst[8];   // where this lane's 16 bytes of its eight rows go in a stage (128-byte swizzle)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = warp * 32 + i * 4 + (lane >> 3);
      dst[i] = (uint32_t)r * TC_KBLOCK_BYTES + (uint32_t)((chunk ^ (r & 7)) << 4);
    }
    // (what a tile is about is looked up while the tile before it is fetched)
    auto lookup = [&](uint32_t tile, int &e, int &place) {
      if (tile >= n_tiles) return;
      const uint32_t m = tile / splits;
      e = p.tile_expert[m];
      if (gather) place = p.order[(int64_t)m * TC_BM + warp * 32 + lane];
    };
    int e_next = 0, place_next = -1;
    lookup(blockIdx.x, e_next, place_next);
    for (uint32_t tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x) {
      const int m = (int)(tile / splits), c0 = (int)(tile % splits) * p.cols_per_tile;
      const int e = e_next, place = place_next;
      lookup(tile + gridDim.x, e_next, place_next);
      const unsigned char *src[8];
      uint32_t real = 0;   // bit i: row i of this lane's has a place
      if (gather) {
        const int row = place < 0 ? -1 : place / p.gather_div;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = __shfl_sync(0xffffffffu, row, i * 4 + (lane >> 3));
          src[i] = reinterpret_cast<const unsigned char *>(p.A) + ((int64_t)(r < 0 ? 0 : r) * p.K) * (EIGHT ? 1 : 2) + chunk * 16;
          real |= (r >= 0 ? 1u : 0u) << i;
        }
      }
      for (int round = 0; round < slices * PASSES && ok; ++round) {
        int pa = 0, pb = 0;
        if constexpr (LONG_SUMS) pass_parts(round % PASSES, &pa, &pb);
        const int kb0 = LONG_SUMS ? round / PASSES * EX_SLICE : 0, kb1 = LONG_SUMS && kb0 + EX_SLICE < p.kb ? kb0 + EX_SLICE : p.kb;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (lane == 0) {
            ok = mbar_wait(&empty[stage], phase ^ 1u, abort_flag, p.spin_limit, EX_TMA_BACKOFF);
            if (ok && warp == 0) mbar_arrive_expect_tx(&full[stage], tma_bytes);
          }
          ok = __shfl_sync(0xffffffffu, (int)ok, 0);
          if (!ok) break;
          unsigned char *to = base + (size_t)stage * stage_bytes;
          if (warp == 0) {
            if (lane >= 8 && lane < 8 + P && !gather) tma_load_2d(to + (lane - 8) * EX_STAGE_A, &map_a, kb * BK, (TRI ? lane - 8 : pa) * p.a_rows + m * TC_BM, &full[stage]);
            unsigned char *to_w = to + P * EX_STAGE_A;
            if (p.box_panels > 0) {   // runs of panels in a copy each
              // gated: the first half of the panels are columns of the gate, the second of what it gates
              constexpr int RUNS = GATED ? 2 : 1;
              if (lane >= 16 && lane < 16 + RUNS * P) {
                const int run = (lane - 16) % RUNS, part = (lane - 16) / RUNS;
                tma_load_4d(to_w + part * b_bytes + run * p.box_panels * PANEL, &map_w, 0, kb * BK, (run ? p.cols + c0 : c0) / BK, (TRI ? part : pb) * p.n_experts + e, &full[stage]);
              }
            } else if (lane >= 16 && lane - 16 < P * p.bn / BK) {   // a panel of the weights a lane
              const int panels = p.bn / BK, part = (lane - 16) / panels, c = (lane - 16) % panels * BK;
              const int col = GATED && c >= p.cols_per_tile ? p.cols + c0 + c - p.cols_per_tile : c0 + c;
              tma_load_3d(to_w + (lane - 16) * PANEL, &map_w, col, kb * BK, (TRI ? part : pb) * p.n_experts + e, &full[stage]);
            }
            __syncwarp();
          }
          if (gather) {
            const uint32_t to_s = smem_u32(to);
            const bool in = kb * TC_KBLOCK_BYTES + chunk * 16 < p.K * (EIGHT ? 1 : 2);   // (rows are multiples of 16 bytes)
#pragma unroll
            for (int i = 0; i < 8; ++i) cp_async16(to_s + dst[i], in ? src[i] + (int64_t)kb * TC_KBLOCK_BYTES : p.A, in && ((real >> i) & 1u) ? 16u : 0u);
            cp_async_arrive(&full[stage]);
          }
          if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; came_round = true; }
        }
      }
    }
    __syncwarp();
    cp_async_wait_all();
    // (after an abort a stage may lack another warp's arrivals: the wait for the copies in flight then ends by its limit)
    if (lane == 0 && warp == 0) ring_drain(full, (uint32_t)p.stages, stage, phase, came_round);
  } else if (warp == EX_MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuer
    // D = fp32, A K-major, B MN-major (bit 16), N = bn, M = 128; operands bf16 (1) or e4m3 (0)
    const uint32_t fmt = EIGHT ? 0u : 1u, lead = lane == 0;
    const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | (1u << 16) | ((uint32_t)(p.bn >> 3) << 17) | ((uint32_t)(TC_BM >> 4) << 24);
    uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
    bool ok = true;
    for (uint32_t tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x)
    for (int slice = 0; slice < slices; ++slice) {
      const int kbs = LONG_SUMS && p.kb - slice * EX_SLICE > EX_SLICE ? EX_SLICE : p.kb - (LONG_SUMS ? slice * EX_SLICE : 0);   // k-blocks of a pass
      ok = ex_wait_warp(&acc_empty[acc], acc_phase ^ 1u, abort_flag, p.spin_limit);
      if (!ok) break;
      tc_fence_after();
      for (int kb = 0; kb < kbs * PASSES; ++kb) {
        ok = ex_wait_warp(&full[stage], phase, abort_flag, p.spin_limit);
        if (!ok) break;
        // gathered rows were written by the threads of the other warps: what follows reads them through the tensor core's path
        if (p.gather_div) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        const uint32_t a_s = smem_u32(base) + stage * (uint32_t)stage_bytes;
        if constexpr (TRI) {
          const uint32_t d_main = tmem_base + acc * acc_stride, d_small = d_main + (uint32_t)p.bn;
#pragma unroll
          for (int pass = 0; pass < 6; ++pass) {
            int pa, pb;
            pass_parts(pass, &pa, &pb);
            const uint64_t a_d = make_desc(a_s + pa * EX_STAGE_A), b_d = make_desc_mn(a_s + 3 * EX_STAGE_A + (uint32_t)(pb * b_bytes), PANEL);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              ex_mma<false>(lead, pass == 5 ? d_main : d_small, a_d + k * 2, b_d + k * (PANEL / 64), idesc, kb > 0 || k != 0 || (pass != 0 && pass != 5));
          }
        } else {
          const uint64_t a_d = make_desc(a_s), b_d = make_desc_mn(a_s + EX_STAGE_A, PANEL);
          const uint32_t d_tmem = tmem_base + acc * acc_stride;
#pragma unroll
          for (int k = 0; k < 4; ++k)   // four steps of 32 bytes of K: a quarter of the k-block's rows of W
            ex_mma<EIGHT>(lead, d_tmem, a_d + k * 2, b_d + k * (PANEL / 64), idesc, kb > 0 || k != 0);
        }
        ex_commit(lead, &empty[stage]);
        if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      ex_commit(lead, &acc_full[acc]);
      if (++acc == bufs) { acc = 0; acc_phase ^= 1u; }
    }
    ex_commit(lead, mma_done);
    mbar_drain(mma_done, 0);
  } else if (warp == EX_META_WARP) {
    // ------------------------------------------------------------------ what the epilogue needs, ahead of it: two loads, one behind the other, for
    // every tile, and four rows and columns a lane.  (Made by the epilogue where it needs them, these waits took most of its time.)
    uint32_t acc = 0, acc_phase = 0;
    int4 place_next = make_int4(-1, -1, -1, -1);
    int e_next = 0;
    auto look = [&](uint32_t tile) {
      if (tile >= n_tiles) return;
      const uint32_t m = tile / splits;
      place_next = *reinterpret_cast<const int4 *>(p.order + (int64_t)m * TC_BM + lane * 4);
      e_next = p.tile_expert[m];
    };
    look(blockIdx.x);
    for (uint32_t tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
      const int4 place = place_next;
      const int64_t w_row = (int64_t)e_next * p.w_cols;
      const int c_tile = (int)(tile % splits) * p.cols_per_tile;
      look(tile + gridDim.x);
      float4 weight = make_float4(1.f, 1.f, 1.f, 1.f), xs = weight, bias[2], scale[2];
      if (STORE == IT_EXPERT_OUT_BF16 || STORE == IT_EXPERT_OUT_F32) {
        weight.x = place.x < 0 ? 0.f : p.weights[place.x]; weight.y = place.y < 0 ? 0.f : p.weights[place.y];
        weight.z = place.z < 0 ? 0.f : p.weights[place.z]; weight.w = place.w < 0 ? 0.f : p.weights[place.w];
      }
      if constexpr (EIGHT) {
        xs.x = place.x < 0 ? 0.f : p.x_scale[place.x / p.x_div]; xs.y = place.y < 0 ? 0.f : p.x_scale[place.y / p.x_div];
        xs.z = place.z < 0 ? 0.f : p.x_scale[place.z / p.x_div]; xs.w = place.w < 0 ? 0.f : p.x_scale[place.w / p.x_div];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {   // columns of the accumulator, four a lane (gated: the second half of them belongs to columns p.cols and on)
        bias[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        scale[i] = make_float4(1.f, 1.f, 1.f, 1.f);
        const int ac = i * 128 + lane * 4, second = GATED && ac >= p.cols_per_tile, c = c_tile + ac - (second ? p.cols_per_tile : 0);
        if (ac >= p.bn || c >= p.cols) continue;
        const int64_t at = w_row + c + (second ? p.cols : 0);
        if (p.bias) bias[i] = *reinterpret_cast<const float4 *>(p.bias + at);
        if constexpr (EIGHT) scale[i] = *reinterpret_cast<const float4 *>(p.w_scale + at);
      }
      if constexpr (LONG_SUMS) {   // (the slices before the last need nothing of this)
        bool ok = true;
        for (int slice = 0; slice + 1 < slices && ok; ++slice) {
          ok = lane == 0 ? mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag, p.spin_limit, EX_EPI_BACKOFF) : true;
          ok = __shfl_sync(0xffffffffu, (int)ok, 0);
          if (ok && lane == 0) mbar_arrive(&meta_full[acc]);
          acc_phase ^= 1u;
        }
        if (!ok) break;
      }
      bool ok = lane == 0 ? mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag, p.spin_limit, EX_EPI_BACKOFF) : true;
      if (!__shfl_sync(0xffffffffu, (int)ok, 0)) break;
      Meta &k = meta[acc];
      *reinterpret_cast<int4 *>(k.place + lane * 4) = place;
      *reinterpret_cast<float4 *>(k.weight + lane * 4) = weight;
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<float4 *>(k.bias + i * 128 + lane * 4) = bias[i];
      if constexpr (EIGHT) {
        *reinterpret_cast<float4 *>(k.xs + lane * 4) = xs;
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<float4 *>(k.scale + i * 128 + lane * 4) = scale[i];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&meta_full[acc]);
      if (++acc == bufs) { acc = 0; acc_phase ^= 1u; }
    }
  } else {
    // ------------------------------------------------------------------ epilogue: a thread per row of the tile, a warp per 32 rows and step of columns
    const int quarter = warp & 3, sub = (warp - EX_EPI_WARP0) >> 2;   // a warp may only touch TMEM lanes [32 * (warp % 4), +32)
    constexpr bool F32_OUT = STORE == IT_EXPERT_SUMS || STORE == IT_EXPERT_OUT_F32, DIRECT = STORE == IT_EXPERT_OUT_BF16 || STORE == IT_EXPERT_OUT_F32;
    constexpr int ESIZE = F32_OUT ? 4 : 2, COLS = 64 / ESIZE;   // 64 bytes of a row are staged at a time
    constexpr int PLANES = STORE == IT_EXPERT_PARTS ? 3 : 1;
    constexpr int ROW = DIRECT ? 128 : 64, PIECES = ROW / 16, AT_ONCE = 32 / PIECES;   // staging tile: bytes of a row, its lanes, rows that a warp stores at once
    const uint32_t stage_s = smem_u32(staging) + (uint32_t)(warp - EX_EPI_WARP0) * ex_staging(STORE);
    // 16-byte pieces are swizzled: this lane's row as it writes it (piece i: put ^ 16 i), and its piece of every row that it stores
    const int row0 = lane / PIECES, piece = lane % PIECES;
    const uint32_t put = stage_s + (uint32_t)lane * ROW + (uint32_t)((DIRECT ? lane & 7 : (lane >> 1) & 3) << 4);
    const uint32_t row8 = 8u * (uint32_t)p.cols * ESIZE;
    const uint32_t floor2 = p.act == IT_ACT_RELU ? 0u : 0xff80ff80u;   // bf16 pair: 0, or minus infinity where nothing is cut off
    uint32_t acc = 0, acc_phase = 0;
    for (uint32_t tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
      const int m = (int)(tile / splits), c_tile = (int)(tile % splits) * p.cols_per_tile;
      if constexpr (LONG_SUMS) {
        // this warp's columns of every slice but the last: into the place of the sums, or added to what is there
        const int cols = p.cols - c_tile < p.cols_per_tile ? p.cols - c_tile : p.cols_per_tile;
        const int half = (cols + 32 * EX_EPI_SUBS - 1) / (32 * EX_EPI_SUBS) * 32, from = sub * half, upto = from + half < cols ? from + half : cols;
        const uint32_t product = tmem_base + ((uint32_t)(quarter * 32) << 16), sums = product + (uint32_t)p.bn;
        bool ok = true;
        for (int slice = 0; slice + 1 < slices; ++slice) {
          ok = mbar_wait(&meta_full[0], acc_phase, abort_flag, p.spin_limit, EX_EPI_BACKOFF) && mbar_wait(&acc_full[0], acc_phase, abort_flag, p.spin_limit, EX_EPI_BACKOFF);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int second = 0; second < (GATED ? 2 : 1); ++second)
            for (int c = from + second * p.cols_per_tile; c < upto + second * p.cols_per_tile; c += 16) {
              uint32_t r[16], q[16];
              tmem_ld16(product + (uint32_t)c, r);
              if (slice > 0) tmem_ld16(sums + (uint32_t)c, q);
              tmem_ld_wait();
              if (slice > 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(q[i]));
              }
              tmem_st16(sums + (uint32_t)c, r);
            }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&acc_empty[0]);
          acc_phase ^= 1u;
        }
        if (!ok) break;
      }
      const int64_t pos0 = (int64_t)m * TC_BM + quarter * 32;
      const bool ok = mbar_wait(&meta_full[acc], acc_phase, abort_flag, p.spin_limit, EX_EPI_BACKOFF) &&
                      mbar_wait(&acc_full[acc], acc_phase, abort_flag, p.spin_limit, EX_EPI_BACKOFF);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const Meta &k = meta[acc];
      uint64_t xs2 = 0, weight2 = 0;
      if constexpr (EIGHT) { const uint32_t x = __float_as_uint(k.xs[quarter * 32 + lane]); xs2 = pack2(x, x); }
      if constexpr (DIRECT) { const uint32_t x = __float_as_uint(k.weight[quarter * 32 + lane]); weight2 = pack2(x, x); }
      unsigned char *to = reinterpret_cast<unsigned char *>(p.dst) + ((DIRECT ? 0 : pos0 + row0) * p.cols + c_tile) * ESIZE + piece * 16;
      uint32_t real = 0;   // rows of this lane that are stored
      if constexpr (!DIRECT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) real |= (k.place[quarter * 32 + 8 * i + row0] >= 0 ? 1u : 0u) << i;
      }
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * acc_stride;
      const int width = p.cols - c_tile < p.cols_per_tile ? p.cols - c_tile : p.cols_per_tile;
      // 64 bytes of this lane's row into the staging tile ...
      auto stage = [&](const uint32_t *w, int half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) st_shared_v4(put ^ (16u * (4 * half + i)), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      };
      // ... and out again as pieces of rows; c: their first column in the tile
      auto flush = [&](int c, int64_t plane, bool both) {
        __syncwarp();
        const bool in = c + piece * (16 / ESIZE) < width && (!DIRECT || both || piece < 4);
#pragma unroll
        for (int i = 0; i < 32 / AT_ONCE; ++i) {
          const int row = AT_ONCE * i + row0;
          const uint32_t from = stage_s + (uint32_t)row * ROW + (uint32_t)((piece ^ (DIRECT ? row & 7 : (row >> 1) & 3)) << 4);
          uint4 d;
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(d.x), "=r"(d.y), "=r"(d.z), "=r"(d.w) : "r"(from) : "memory");
          if constexpr (DIRECT) {
            const int at = k.place[quarter * 32 + row];
            if (in && at >= 0) *reinterpret_cast<uint4 *>(to + ((int64_t)at * p.cols + c) * ESIZE) = d;
          } else {
            if (in && ((real >> i) & 1u)) *reinterpret_cast<uint4 *>(to + (uint64_t)i * row8 + (plane + c) * ESIZE) = d;
          }
        }
        __syncwarp();
      };
      // this warp's columns: one half of the tile's, so that what it writes of a row lies together
      const int half_cols = (width + 32 * EX_EPI_SUBS - 1) / (32 * EX_EPI_SUBS) * 32, lo = sub * half_cols, hi = lo + half_cols < width ? lo + half_cols : width;
      // 32 columns of the accumulator (gated: and of what they gate), from c on
      auto finish = [&](const uint32_t (&r)[32], const uint32_t (&r2)[GATED ? 32 : 1], int c) {
        uint64_t v[16];
        auto scaled = [&](const uint32_t *acc_r, int at, uint64_t *o) {
          const ulonglong2 *b = reinterpret_cast<const ulonglong2 *>(k.bias + at);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const ulonglong2 bb = b[i];
            uint64_t lo = pack2(acc_r[4 * i], acc_r[4 * i + 1]), hi = pack2(acc_r[4 * i + 2], acc_r[4 * i + 3]);
            if constexpr (EIGHT) {
              const ulonglong2 f = reinterpret_cast<const ulonglong2 *>(k.scale + at)[i];
              lo = fma2(mul2(lo, xs2), f.x, bb.x);
              hi = fma2(mul2(hi, xs2), f.y, bb.y);
            } else {
              lo = add2(lo, bb.x);
              hi = add2(hi, bb.y);
            }
            o[2 * i] = lo;
            o[2 * i + 1] = hi;
          }
        };
        scaled(r, c, v);
        constexpr bool CUT_LATER = !F32_OUT && !GATED && !DIRECT && STORE != IT_EXPERT_PARTS;   // ReLU on the rounded pairs
        if (!CUT_LATER || p.act != IT_ACT_RELU) expert_act(v, p.act);
        if constexpr (GATED) {
          uint64_t u[16];
          scaled(r2, p.cols_per_tile + c, u);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = mul2(v[i], u[i]);
        }
        if constexpr (DIRECT) {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = mul2(v[i], weight2);
        }
        if constexpr (F32_OUT) {
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 f = unpack2(v[i]);
            w[2 * i] = __float_as_uint(f.x); w[2 * i + 1] = __float_as_uint(f.y);
          }
          if constexpr (DIRECT) {
            stage(w, 0);
            stage(w + 16, 1);
            flush(c, 0, true);
          } else {
            stage(w, 0);
            flush(c, 0, false);
            if (c + COLS < width) {
              stage(w + 16, 0);
              flush(c + COLS, 0, false);
            }
          }
        } else if constexpr (STORE == IT_EXPERT_PARTS) {
          constexpr uint64_t MINUS = 0xbf800000bf800000ull;   // (-1, -1)
#pragma unroll
          for (int pl = 0; pl < PLANES; ++pl) {   // the upper halves, then what they leave
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 f = unpack2(v[i]);
              const uint32_t lo = __float_as_uint(f.x), hi = __float_as_uint(f.y);
              w[i] = __byte_perm(lo, hi, 0x7632);
              if (pl < 2) v[i] = fma2(pack2(lo & 0xffff0000u, hi & 0xffff0000u), MINUS, v[i]);
            }
            stage(w, 0);
            flush(c, pl * p.part_stride, false);
          }
        } else {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 f = unpack2(v[i]);
            w[i] = bf16x2_of(f.x, f.y);
            if constexpr (CUT_LATER) w[i] = max_bf16x2(w[i], floor2);
          }
          if constexpr (DIRECT) {
            const int half = ((c - lo) >> 5) & 1;
            stage(w, half);
            if (half == 1 || c + 32 >= hi) flush(c - 32 * half, 0, half == 1);
          } else {
            stage(w, 0);
            flush(c, 0, false);
          }
        }
      };
      // (the next 32 columns read ahead would take registers that are not there: with them spilled the epilogue took twice as long)
      auto read = [&](int col, uint32_t (&r)[32]) {
        tmem_ld32(taddr + (uint32_t)col, r);
        if constexpr (TRI || LONG_SUMS) {
          uint32_t q[32];
          tmem_ld32(taddr + (uint32_t)(p.bn + col), q);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(q[i]));
        } else {
          tmem_ld_wait();
        }
      };
      uint32_t r[32], r2[GATED ? 32 : 1];
      for (int c = lo; c < hi; c += 32) {
        read(c, r);
        if constexpr (GATED) read(p.cols_per_tile + c, r2);
        finish(r, r2, c);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[acc]);
      if (++acc == bufs) { acc = 0; acc_phase ^= 1u; }
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.status, 1);
  if (warp == EX_MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem_base, tmem_cols);
  }
}

// ----------------------------------------------------------------------------- host side
template <bool EIGHT, it_expert_store STORE, bool GATED, ExForm FORM = EX_PLAIN>
it_status launch(const CUtensorMap &ma, const CUtensorMap &mw, const ExParams &p, int grid, int smem, double bytes, double flops, cudaStream_t st) {
  IT_CUDA_TRY(cudaFuncSetAttribute(expert_gemm_kernel<EIGHT, STORE, GATED, FORM>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  IT_LAUNCH(IT_K_EXPERT_GEMM, bytes, flops, st, IT_CUDA_TRY(it_launch_pdl(expert_gemm_kernel<EIGHT, STORE, GATED, FORM>, dim3((unsigned)grid), dim3(EX_THREADS), smem, st, ma, mw, p)));
  return IT_OK;
}

}  // namespace

it_status it_launch_expert_gemm(const it_experts_args &a, const it_experts_plan &q, const it_expert_gemm &g, cudaStream_t st) {
  const int elem = g.eight ? 1 : 2, BK = TC_KBLOCK_BYTES / elem;
  ExParams p{};
  p.order = q.order; p.tile_expert = q.tile_expert; p.n_tiles = q.n_tiles; p.tiles_max = (int)q.tiles_max;
  p.K = g.K; p.kb = (g.K + BK - 1) / BK;
  p.A = g.A; p.gather_div = g.gather ? a.d.top_k : 0; p.a_rows = (int)g.a_rows;
  p.n_experts = a.d.n_experts; p.w_cols = g.w_cols; p.cols = g.cols; p.act = g.act; p.gated = g.gated;
  p.bias = g.bias; p.w_scale = g.w_scale; p.x_scale = g.x_scale; p.weights = a.weights; p.x_div = a.d.top_k;
  p.dst = g.dst; p.part_stride = q.tiles_max * TC_BM * (int64_t)g.cols; p.status = a.status;
  p.spin_limit = g.spin_limit ? g.spin_limit : TC_SPIN_LIMIT; p.no_loads = g.no_loads;
  // fp32: with the parts of a k-block in one stage they are fetched once instead of twice each, and the six products are issued behind one wait; two stages
  // and the second accumulator leave 128 columns (64 where rows are stored 128 bytes at a time).
  const bool tri = g.parts == 3 && g.K <= EX_SLICE * 64;
  // columns in as few tiles as 256 accumulator columns allow, of equal width in whole panels
  const int most = (tri ? (ex_direct(g.store) ? 64 : 128) : 256) / (g.gated ? 2 : 1);
  p.n_splits = (g.cols + most - 1) / most;
  p.cols_per_tile = ((g.cols + p.n_splits - 1) / p.n_splits + BK - 1) / BK * BK;
  p.n_splits = (g.cols + p.cols_per_tile - 1) / p.cols_per_tile;
  p.bn = g.gated ? 2 * p.cols_per_tile : p.cols_per_tile;
  // A tensor core cuts off what it adds to an accumulator, which pulls long sums towards zero: fp32, 2-norm of the error with one accumulator for all of K =
  // 256, 512, 1024, 2048 2.5e-7, 4.9e-7, 9.8e-7, 2.1e-6 (a library's fp32 product 2.9e-7 to 7e-7), and in proportion; where products follow one another, and in the two
  // factors of a gate, it adds up (512-1024-512 gated, in slices of 512, 1.4e-6, plain fp32 8.1e-7).  Above K = 256 the epilogue adds up slices of 256, rounding to nearest:
  // 2.6e-7 for K = 512 to 4096, 512-1024-512 gated 7.7e-7.  Against slices of 512 and TRI up to there: 40k x 512 x 256 140 us / 142, 40k x 1024 x 256 256 / 252,
  // 20k, 2 of 4, 256-1024-256 325 / 322, gated 512-1024-512 812 / 722, 128-512-128 144 / 117.  (Slices of 128, 1.7e-7: 143, 264, 331, 838, 146.)

  const cuuint64_t da[2] = {(cuuint64_t)g.K, (cuuint64_t)(g.a_rows * g.parts)}, sa[1] = {(cuuint64_t)g.K * elem};
  const cuuint32_t ba[2] = {(cuuint32_t)BK, (cuuint32_t)TC_BM};
  CUtensorMap ma, mw;
  IT_TRY(encode(&ma, g.eight, g.A, 2, da, sa, ba));
  // Columns in whole panels: W as [experts][panels][K][panel's columns], of which one copy fetches what a tile takes of a k-block (gated: of
  // either half).  Otherwise a copy per panel, which fills what lies beyond a row with zeros.
  const cuuint64_t n_mats = (cuuint64_t)a.d.n_experts * g.parts, row = (cuuint64_t)g.w_cols * elem;
  p.box_panels = 0;
  if (g.w_cols % BK == 0 && g.cols % BK == 0) {
    p.box_panels = (g.gated ? p.cols_per_tile : p.bn) / BK;
    const cuuint64_t dw[4] = {(cuuint64_t)BK, (cuuint64_t)g.K, (cuuint64_t)(g.w_cols / BK), n_mats}, sw[3] = {row, TC_KBLOCK_BYTES, row * (cuuint64_t)g.K};
    const cuuint32_t bw[4] = {(cuuint32_t)BK, (cuuint32_t)BK, (cuuint32_t)p.box_panels, 1};
    IT_TRY(encode(&mw, g.eight, g.W, 4, dw, sw, bw));
  } else {
    const cuuint64_t dw[3] = {(cuuint64_t)g.w_cols, (cuuint64_t)g.K, n_mats}, sw[2] = {row, row * (cuuint64_t)g.K};
    const cuuint32_t bw[3] = {(cuuint32_t)BK, (cuuint32_t)BK, 1};
    IT_TRY(encode(&mw, g.eight, g.W, 3, dw, sw, bw));
  }

  const int stage = (tri ? 3 : 1) * (EX_STAGE_A + p.bn * TC_KBLOCK_BYTES), fixed = EX_EPI_WARPS * ex_staging(g.store) + 2 * (int)(g.eight ? sizeof(ExMetaEight) : sizeof(ExMeta)) + (2 * EX_MAX_STAGES + 9) * 8;
  p.stages = (227 * 1024 - fixed) / stage;
  if (p.stages > EX_MAX_STAGES) p.stages = EX_MAX_STAGES;
  const int smem = fixed + p.stages * stage;
  const int64_t tiles = q.tiles_max * p.n_splits;
  IT_REQUIRE(tiles + 3 * (int64_t)a.sms <= INT32_MAX, IT_ERR_UNSUPPORTED, "too many places and columns for one launch");
  const int grid = (int)(tiles < a.sms ? tiles : a.sms);
  const int64_t places = a.n * a.d.top_k;
  const double flops = 2.0 * places * g.K * (double)g.w_cols, bytes = (double)places * (g.K * elem * g.parts + g.cols * 4.0);
#define IT_EX_LAUNCH(EIGHT, STORE, GATED) return launch<EIGHT, STORE, GATED>(ma, mw, p, grid, smem, bytes, flops, st)
#define IT_EX_F32(STORE, GATED)                                                                 \
  if (tri) return launch<false, STORE, GATED, EX_TRI>(ma, mw, p, grid, smem, bytes, flops, st); \
  return launch<false, STORE, GATED, EX_LONG_SUMS>(ma, mw, p, grid, smem, bytes, flops, st)
  switch (g.store) {
    case IT_EXPERT_HIDDEN:
      if (g.eight) { if (g.gated) IT_EX_LAUNCH(true, IT_EXPERT_HIDDEN, true); else IT_EX_LAUNCH(true, IT_EXPERT_HIDDEN, false); }
      if (g.gated) IT_EX_LAUNCH(false, IT_EXPERT_HIDDEN, true);
      IT_EX_LAUNCH(false, IT_EXPERT_HIDDEN, false);
    case IT_EXPERT_PARTS:
      if (g.gated) { IT_EX_F32(IT_EXPERT_PARTS, true); }
      IT_EX_F32(IT_EXPERT_PARTS, false);
    case IT_EXPERT_SUMS:
      if (g.eight) IT_EX_LAUNCH(true, IT_EXPERT_SUMS, false);
      if (g.parts == 3) { IT_EX_F32(IT_EXPERT_SUMS, false); }
      IT_EX_LAUNCH(false, IT_EXPERT_SUMS, false);
    case IT_EXPERT_OUT_BF16:
      if (g.eight) IT_EX_LAUNCH(true, IT_EXPERT_OUT_BF16, false);
      IT_EX_LAUNCH(false, IT_EXPERT_OUT_BF16, false);
    default:
      IT_EX_F32(IT_EXPERT_OUT_F32, false);
  }
#undef IT_EX_F32
#undef IT_EX_LAUNCH
}
