// The gated half of a feed-forward block, forward and backward (non-attention work of a layer, paper Sec. 4.1.2), on the
// 5th-generation tensor cores.
//     forward   g = x Wg^T, u = x Wu^T, h = act(g) u, from one pass over x: the tile of g and the tile of u of the same columns are
//               one accumulator, side by side, and the activation and the product are its epilogue
//     backward  dg = dh u act'(g), du = dh act(g) (one elementwise pass, rounded to bf16: they are operands of products next);
//               dWg = dg^T x, dWu = du^T x, dx = dg Wg + du Wu, all three in one launch
// 4 T d f flop there and 8 T d f back: bound by the tensor cores from some hundred tokens on, below by the bytes of the weights.
//
// Products. A pair of CTAs (tcgen05 cta_group::2) computes tiles of 256 or 512 rows x 2 `nh` columns: each CTA loads its own rows of A
// and its own nh rows of B by TMA, so that a byte of either operand is staged once for the two SMs that use it. In the forward pass
// the first CTA's part of B comes from Wg and the second one's from Wu. Operands whose contraction index is not the contiguous one
// (dg^T, du^T, x, and the weights of dx) are read MN-major by the tensor core: nothing is transposed in memory.
//   flat tiles, 256 rows: the accumulators in TMEM are double-buffered, 256 columns of the next tile are filled while the epilogue
//     drains the last one's.
//   tall tiles, 512 rows: two products share a stage of B, their accumulators fill TMEM, and the next tile's first products wait
//     for the epilogue to read the first half; up to four stages of them are issued before the second half is needed. A quarter
//     less to load for the same products.
// A stage of an operand is one instruction of one warp: a 3-D box is several blocks of 64 columns at once. With stages of 64 steps
// and boxes of 64 columns the kernel was bound by the number of TMA instructions a thread issues (16,384 tokens, 4,096 x 12,288: 2,700
// us there and 7,000 back; boxes of 128 columns 2,670 and 5,790; stages of 128 steps 2,390 and 4,840).
#include <atomic>
#include <cmath>
#include <cstdint>
#include <mutex>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "nsp_internal.cuh"
#include "sm100_ptx.cuh"

namespace nsp {
namespace {

// A stage: kDepth steps of the contraction, of kRows rows of A and up to 128 of B.
template <bool kTall>
struct Geometry {
  static constexpr int kDepth = kTall ? 64 : 128, kStages = kTall ? 4 : 3;  // stages of full operands
  static constexpr int kHalves = kTall ? 2 : 1;  // products of 256 rows a stage of B is used for
  static constexpr int kRows = 128 * kHalves;
  static constexpr uint32_t kBytesA = kRows * kDepth * 2, kBytesB = 128 * kDepth * 2;
};
constexpr uint32_t kOperands = 3 * 64 * 1024;
constexpr int kMostStages = 8;
static_assert(Geometry<true>::kStages * (Geometry<true>::kBytesA + Geometry<true>::kBytesB) == kOperands, "stages");
static_assert(Geometry<false>::kStages * (Geometry<false>::kBytesA + Geometry<false>::kBytesB) == kOperands, "stages");
constexpr uint32_t kBlock = 128 * 64 * 2;  // bytes of a block of 128 rows x 64 columns
constexpr int kThreads = 384;              // producer of A, issuer, producer of B, an idle warp, two warpgroups of epilogue
constexpr int kGroupM = 8, kGroupTall = 4; // row tiles that are walked together (see tile_at)
constexpr int kMostMaps = 20, kMostProblems = 3;

struct Problem {
  int32_t tiles_m, tiles_n, first_tile;
  int32_t segments, k_iters, depth;  // the contraction: `segments` pairs of operands, each of `depth` steps in k_iters stages
  int32_t a_map[2], b_map[2][2];     // [segment], [segment][rank of the CTA]: first of an operand's two maps
  int32_t a_mn, b_mn;                // 1: the contiguous index is the row / column one
  int32_t b_shared;                  // 1: both CTAs' parts of B come from one matrix, nh columns apart
  int32_t splits, per_split, part;   // a tile's contraction in `splits` parts of per_split stages, partial tiles from `part` on
  int32_t rows, cols;                // of the output
  int32_t out_map;                   // forward: of h, g, u
  __nv_bfloat16* out[3];
  int64_t ld[3];
};

// Which tiles a pair computes, in turn. The n_long long ones come first, one after the other to all pairs; the pairs that have one
// less of them (those from `heavy` on) take the next `ahead` rounds of the short ones alone, and the rounds after that begin at
// pair `start`.
struct Schedule {
  int32_t n_long, n_short, heavy, ahead, start;
  __host__ __device__ __forceinline__ int tile(int i, int pair, int pairs) const {  // -1: no more
    const int mine = n_long / pairs + (pair < heavy ? 1 : 0);
    if (i < mine) return pair + i * pairs;
    const int round = i - mine + (pair < heavy ? ahead : 0), light = pairs - heavy;
    int t;
    if (round < ahead) {
      t = round * light + pair - heavy;
    } else {
      int at = pair - start;
      if (at < 0) at += pairs;
      t = ahead * light + (round - ahead) * pairs + at;
    }
    return t < n_short ? n_long + t : -1;
  }
};

struct GemmArgs {
  Problem p[kMostProblems];
  int32_t n_problems, nh;
  // Rows of a box of a K-major A and steps of a box of MN-major operands: 128 and a stage's depth, or fewer where there are no more
  // rows or steps; what the tensor core reads beyond them are other bytes of shared memory, for rows that are not stored. Bytes of a
  // stage of A and of B, and how many stages fit.
  int32_t a_rows, mn_steps, bytes_a, bytes_b, stages;
  Schedule order;
  StatusWord status;
  // SM clocks a wait for operands may take before it gives up; the waits for another role's work may take twice that, so that the
  // record names the load and not what stands behind it
  long long wait_limit;
  int32_t withhold;      // checked build only: the load the second CTA leaves out (1: A, 2: B; failure-detection test), or 0
  float* partial;  // [partial tile][CTA][4 columns][128 rows][4]: accumulators of tiles whose contraction is split
};

struct Maps {
  CUtensorMap m[kMostMaps];
};

struct Smem {
  uint8_t operands[kOperands];  // stages of A, then of B
  uint8_t out[2][kBlock];       // a warpgroup's block of an output on its way to memory
  uint64_t full[kMostStages];   // in the first CTA: the bytes of both
  uint64_t empty[kMostStages];  // in both: the products of the stage have completed
  uint64_t acc_full[2];         // in both: an accumulator is complete (tall tiles: both halves, the first barrier)
  uint64_t acc_empty[2];        // in the first CTA: 16 warps have read it
  uint32_t tmem_base;
  int32_t abort;
};
static_assert(sizeof(Smem) <= 232448, "shared memory budget (227 KB)");

enum Act : int32_t { kSilu = NSP_ACT_SILU, kGelu = NSP_ACT_GELU };

// act(x), and its slope; exp is CUDA's. The normal distribution function at -t, t >= 0, is exp(-t^2 / 2) times a smooth function that falls
// from 1/2 as 1 / t: s times a polynomial in s = 1 / (1 + 0.31 t), fitted for the smallest relative error by reweighted least squares
// (1.7e-7; 4.7e-7 with the roundings of fp32, and t^2 / 2 ulp of the exponential). The slope needs the same exponential. (4,099 x 5,512
// backward: 61 us with erfc and an exponential of its own, 40 so; 16,384 x 12,288 forward, in the epilogue: 2,256 and 2,220.)
__device__ __forceinline__ float normal_cdf(float x, float bell) {  // bell: exp(-x^2 / 2)
  const float s = __fdividef(1.f, fmaf(0.31f, fabsf(x), 1.f));
  float q = fmaf(s, 0.0358906873f, -0.141819388f);
  q = fmaf(q, s, 0.155459404f);
  q = fmaf(q, s, -0.0152864568f);
  q = fmaf(q, s, 0.110326536f);
  q = fmaf(q, s, 0.107700795f);
  q = fmaf(q, s, 0.124072447f);
  q = fmaf(q, s, 0.123656064f);
  const float tail = bell * s * q;
  return x > 0.f ? 1.f - tail : tail;
}
template <int kAct>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (kAct == kSilu) return __fdividef(x, 1.f + __expf(-x));
  return x * normal_cdf(x, __expf(-0.5f * x * x));
}
template <int kAct>
__device__ __forceinline__ void act_both(float x, float& value, float& slope) {
  if constexpr (kAct == kSilu) {
    const float p = __fdividef(1.f, 1.f + __expf(-x));
    value = x * p;
    slope = p * (1.f + x * (1.f - p));
  } else {
    const float bell = __expf(-0.5f * x * x), p = normal_cdf(x, bell);
    value = x * p;
    slope = fmaf(x * 0.39894228040143268f, bell, p);
  }
}

// The tiles of a problem, the parts of a tile one after the other: kGroup row tiles at a time, over all column tiles, so that the tiles under way at one time share
// both their rows and their columns in L2.
template <int kGroup>
__device__ __forceinline__ void tile_at(const Problem& p, int tile, int& m, int& n) {
  tile /= p.splits;
  const int per_group = kGroup * p.tiles_n, group = tile / per_group, rest = tile - group * per_group;
  const int first = group * kGroup, size = min(kGroup, p.tiles_m - first);
  n = rest / size;
  m = first + rest - n * size;
}

__device__ __forceinline__ void tma_load_2d_pair(void* smem_dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}

__device__ __forceinline__ void tma_store_2d(const void* tmap, const void* smem_src, int32_t c0, int32_t c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(smem_src)), "r"(c0), "r"(c1)
               : "memory");
}

// One operand of a stage. `across` is the index of its rows (columns of the output for B), `k` the step of the contraction, `wide` and
// `steps` the box's extent in them. maps[0] holds whole blocks of 64 contiguous columns, two of them (or more) a box: {64, the other
// index, blocks}; maps[1] is the plain matrix, for boxes that the end of the contiguous index cuts: the rest reads as zero.
template <int kDepth>
__device__ __forceinline__ void load_operand(uint8_t* dst, const CUtensorMap* maps, uint32_t bar, int mn, int across, int k, int wide, int steps,
                                             int across_end, int k_end) {
  const int at = mn ? across : k, other = mn ? k : across, end = mn ? across_end : k_end, cols = mn ? wide : kDepth;
  if (at + cols <= end) {
    tma_load_3d_pair(dst, maps, bar, 0, other, at / 64);
  } else {
    const uint32_t block = (mn ? steps : wide) * 128;
    const int last = mn ? cols : min(cols, end - at);  // the contraction ends in this stage: no blocks behind it
    for (int c = 0; c < last; c += 64) tma_load_2d_pair(dst + c / 64 * block, maps + 1, bar, at + c, other);
  }
}
// The stages of one part of a tile's contraction.
struct Part {
  int first, last;
  __device__ __forceinline__ Part(const Problem& p, int tile) {
    const int all = p.segments * p.k_iters;
    first = tile % p.splits * p.per_split;
    last = min(first + p.per_split, all);
  }
};

template <int kDepth>
__device__ __forceinline__ uint32_t operand_bytes(int mn, int wide, int steps, int k, int k_end) {
  return mn ? wide * steps * 2 : k + 64 < k_end ? wide * kDepth * 2 : wide * 64 * 2;
}

// 32 columns of one row
__device__ __forceinline__ void store_row(__nv_bfloat16* out, int64_t ld, int row, int col, int rows, int cols, const uint32_t (&w)[16]) {
  if (row >= rows) return;
  __nv_bfloat16* p = out + row * ld + col;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (col + 8 * i < cols) *reinterpret_cast<uint4*>(p + 8 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// A warpgroup's block of 128 rows x 64 columns, every thread a row, on its way through shared memory (the layout that a TMA store
// with 128-byte swizzle takes): a warp that stores its 32 rows directly touches 32 lines with every instruction.
struct BlockOut {
  uint8_t* stage;
  int wg, thread;
  __device__ __forceinline__ void sync() const { asm volatile("bar.sync %0, 128;" ::"r"(1 + wg) : "memory"); }
  __device__ __forceinline__ bool all(bool here) const {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, %2, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(static_cast<uint32_t>(here)), "r"(1 + wg)
        : "memory");
    return r != 0;
  }
  __device__ __forceinline__ void begin() const {  // the block before has been read
    if (thread == 0) tma_store_wait_read();
    sync();
  }
  __device__ __forceinline__ void put(int c, const uint32_t (&w)[16]) const {  // columns 32 c .. 32 c + 31
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint4*>(stage + thread * 128 + (((4 * c + i) ^ (thread & 7)) * 16)) =
          make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
  __device__ __forceinline__ void end(const CUtensorMap* map, int col, int row0, const Problem& p) const {
    fence_proxy_async_smem();
    sync();
    if (thread == 0 && col < p.cols && row0 < p.rows) {
      tma_store_2d(map, stage, col, row0);
      tma_store_commit();
    }
  }
};

__device__ __forceinline__ void pack_row(const uint32_t (&r)[32], uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
}

// kAct < 0: the accumulator is the output; otherwise the forward pass with that activation
template <int kAct, bool kTall>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) glu_gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ GemmArgs a) {
  using G = Geometry<kTall>;
  constexpr int kDepth = G::kDepth, kTileRows = 2 * G::kRows, kGroup = kTall ? kGroupTall : kGroupM;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem& s = *reinterpret_cast<Smem*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  if (tid == 0) {
    for (int i = 0; i < kMostStages; ++i) mbar_init(&s.full[i], 1), mbar_init(&s.empty[i], 1);
    for (int i = 0; i < 2; ++i) mbar_init(&s.acc_full[i], 1), mbar_init(&s.acc_empty[i], 16);
    s.abort = 0;
    fence_mbar_init();
  }
  __syncwarp();
  if (warp == 0) tmem_alloc_pair(&s.tmem_base, 512);
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();  // both CTAs run and their barriers are initialised
  tc_fence_after_sync();
  grid_wait_predecessor();
  grid_launch_dependents();
  const uint32_t lead = cluster_addr(smem_raw, 0), peer = cluster_addr(smem_raw, rank ^ 1);
  auto off = [&](const void* p) -> uint32_t { return smem_u32(p) - smem_u32(smem_raw); };
  volatile int32_t* abort_flag = &s.abort;
  auto raise_abort = [&]() {
    *abort_flag = 1;
    cluster_store(peer + off(&s.abort), 1);
  };
  const bool misaligned = (smem_u32(smem_raw) & 1023u) != 0;
  if ((misaligned || s.tmem_base != 0) && tid == 0) {
    report_timeout(a.status, -1, kWhereGluSetup, static_cast<int32_t>(s.tmem_base));
    raise_abort();
  }
  const int pairs = static_cast<int>(gridDim.x) / 2, pair = static_cast<int>(blockIdx.x) / 2;
  const int nh = a.nh;
  const int stages = a.stages;
  auto stage_a = [&](uint32_t st) { return s.operands + st * a.bytes_a; };
  auto stage_b = [&](uint32_t st) { return s.operands + stages * a.bytes_a + st * a.bytes_b; };
  struct Turn {  // a stage of the ring and the phase of its barriers
    uint32_t st = 0, ph = 0;
    __device__ __forceinline__ void next(int stages) {
      if (++st == static_cast<uint32_t>(stages)) st = 0, ph ^= 1;
    }
  };
  auto problem_of = [&](int tile) -> const Problem& {
    int k = 0;
    while (k + 1 < a.n_problems && tile >= a.p[k + 1].first_tile) ++k;
    return a.p[k];
  };

  if (warp == 0 || warp == 2) {
    // ================================================================ TMA producers of A and of B (both CTAs, each its own rows)
    if (lane == 0) {
      const bool is_a = warp == 0;
      Turn turn;
      bool ok = true;
      for (int i = 0, tile; ok && (tile = a.order.tile(i, pair, pairs)) >= 0; ++i) {
        const Problem& p = problem_of(tile);
        int m, n;
        tile_at<kGroup>(p, tile - p.first_tile, m, n);
        // first row of A and column of B of either CTA; one whose rows or columns lie behind the end loads nothing
        auto row_of = [&](int r) { return m * kTileRows + r * G::kRows; };
        auto col_of = [&](int r) { return p.b_shared ? n * 2 * nh + r * nh : n * nh; };
        const int mine = static_cast<int>(rank);
        const int across = is_a ? row_of(mine) : col_of(mine), end = is_a ? p.rows : p.cols;
        const int mn = is_a ? p.a_mn : p.b_mn, wide_a = p.a_mn ? G::kRows : a.a_rows, wide = is_a ? wide_a : nh;
        const int of_a = (row_of(0) < p.rows) + (row_of(1) < p.rows), of_b = (col_of(0) < p.cols) + (col_of(1) < p.cols);
        const CUtensorMap* const map0 = &maps.m[is_a ? p.a_map[0] : p.b_map[0][mine]];
        const CUtensorMap* const map1 = &maps.m[is_a ? p.a_map[1] : p.b_map[1][mine]];  // of the second segment
        const Part part(p, tile - p.first_tile);
        for (int k = part.first; k < part.last; ++k, turn.next(stages)) {
          if (*abort_flag || !mbar_wait(&s.empty[turn.st], turn.ph ^ 1, 2 * a.wait_limit)) {
            if (!*abort_flag) report_timeout(a.status, tile, kWhereGluEmpty, k);
            raise_abort();
            ok = false;
            break;
          }
          const bool second = k >= p.k_iters;
          const int at = (second ? k - p.k_iters : k) * kDepth;
          if (is_a && rank == 0)
            mbar_expect_tx(&s.full[turn.st], of_a * operand_bytes<kDepth>(p.a_mn, wide_a, a.mn_steps, at, p.depth) +
                                                 of_b * operand_bytes<kDepth>(p.b_mn, nh, a.mn_steps, at, p.depth));
          bool loads = across < end;
#ifdef NSP_CHECKED
          if (a.withhold == (is_a ? 1 : 2) && rank == 1 && tile == 0 && k == part.first + 1) loads = false;  // never arrives
#endif
          if (loads)
            load_operand<kDepth>(is_a ? stage_a(turn.st) : stage_b(turn.st), second ? map1 : map0, lead + off(&s.full[turn.st]), mn, across, at,
                                 wide, a.mn_steps, end, p.depth);
        }
      }
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ================================================================ issuer of the products, for both CTAs
    const bool leader = elect_one();
    const uint32_t hi = static_cast<uint32_t>(make_smem_desc_sw128(0, 16, 1024) >> 32);
    Turn turn_in;  // of the stage issued next
    uint32_t n_done = 0;
    bool ok = true;
    for (int tile; ok && (tile = a.order.tile(static_cast<int>(n_done), pair, pairs)) >= 0; ++n_done) {
      const Problem& p = problem_of(tile);
      const uint32_t buf = kTall ? 0 : n_done & 1, turn = kTall ? n_done & 1 : (n_done >> 1) & 1;
      const uint32_t idesc = make_idesc_bf16(256, 2 * nh, p.a_mn, p.b_mn);
      // 16 steps of the contraction: 32 bytes of a row (four of them in a block), or 16 rows
      const uint32_t mn_block = a.mn_steps * 8;  // in units of 16 bytes: 64 columns of an MN-major operand
      const uint32_t a_lbo = (p.a_mn ? mn_block : 1u) << 16, a_step = p.a_mn ? 128 : 2, a_next = p.a_mn ? 512 : a.a_rows * 8;
      const uint32_t a_half = p.a_mn ? 2 * mn_block : kBlock >> 4;  // 128 rows on
      const uint32_t b_lbo = (p.b_mn ? mn_block : 1u) << 16, b_step = p.b_mn ? 128 : 2, b_next = p.b_mn ? 512 : nh * 8;
      const Part part(p, tile - p.first_tile);
      const int iters = part.last - part.first;
      auto acc_free = [&](uint32_t which) -> bool {
        const bool here = cluster_wait_tmem(&s.acc_empty[which], turn ^ 1, 2 * a.wait_limit);
        if (!__all_sync(0xffffffffu, here)) {
          if (lane == 0) report_timeout(a.status, tile, kWhereGluAccEmpty, static_cast<int32_t>(which)), raise_abort();
          return false;
        }
        tc_fence_after_sync();
        return true;
      };
      auto arrived = [&](int k, const Turn& at) -> bool {
        const bool here = *abort_flag == 0 && cluster_wait(&s.full[at.st], at.ph, a.wait_limit);
        if (!__all_sync(0xffffffffu, here)) {
          if (lane == 0 && !*abort_flag) report_timeout(a.status, tile, kWhereGluFull, k);
          if (lane == 0) raise_abort();
          return false;
        }
        tc_fence_after_sync();
        return true;
      };
      auto issue = [&](int k, uint32_t st, uint32_t half, bool last_use) {
        const int at = part.first + k;
        const int left = p.depth - (at >= p.k_iters ? at - p.k_iters : at) * kDepth;  // steps of the segment from this stage on
        if (leader) {
          const uint32_t a_lo = (smem_desc_addr(stage_a(st)) + half * a_half) | a_lbo, b_lo = smem_desc_addr(stage_b(st)) | b_lbo;
#pragma unroll
          for (int kk = 0; kk < kDepth / 16; ++kk) {
            if (kk * 16 < left)
              umma2_ss_lh((buf + half) * 256, a_lo + (kk >> 2) * a_next + (kk & 3) * a_step, hi, b_lo + (kk >> 2) * b_next + (kk & 3) * b_step,
                          hi, idesc, (k | kk) != 0);
          }
          if (last_use) umma2_commit(&s.empty[st]);
          if (last_use && k + 1 == iters) umma2_commit(&s.acc_full[buf]);
        }
        __syncwarp();
      };
      ok = acc_free(buf);
      int k = 0;
      if constexpr (kTall) {
        const int lead_in = min(stages, iters);
        Turn ahead = turn_in;
        for (; ok && k < lead_in; ++k, ahead.next(stages)) {
          ok = arrived(k, ahead);
          if (ok) issue(k, ahead.st, 0, false);
        }
        ok = ok && acc_free(1);
        if (ok) {
          for (k = 0; k < lead_in; ++k, turn_in.next(stages)) issue(k, turn_in.st, 1, true);
        }
      }
      for (; ok && k < iters; ++k, turn_in.next(stages)) {
        ok = arrived(k, turn_in);
        if (!ok) break;
        issue(k, turn_in.st, 0, !kTall);
        if constexpr (kTall) issue(k, turn_in.st, 1, true);
      }
    }
  } else if (warp >= 4) {
    // ================================================================ epilogue: a warpgroup has half of the columns
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    uint32_t n_done = 0;
    for (int tile; (tile = a.order.tile(static_cast<int>(n_done), pair, pairs)) >= 0; ++n_done) {
      const Problem& p = problem_of(tile);
      int m, n;
      tile_at<kGroup>(p, tile - p.first_tile, m, n);
      const uint32_t buf0 = kTall ? 0 : n_done & 1, turn = kTall ? n_done & 1 : (n_done >> 1) & 1;
      const bool here = *abort_flag == 0 && mbar_wait(&s.acc_full[buf0], turn, 2 * a.wait_limit);
      const int thread = quad * 32 + lane;
      const BlockOut out{s.out[half], half, thread};
      if (!out.all(here)) {  // the warpgroup goes on together: it meets at barriers below
        if (lane == 0 && !here && !*abort_flag) report_timeout(a.status, tile, kWhereGluAccFull, 0);
        if (lane == 0) raise_abort();
        break;
      }
      tc_fence_after_sync();
#pragma unroll 1
      for (int j = 0; j < G::kHalves; ++j) {
      const uint32_t buf = buf0 + j;
      const int row0 = m * kTileRows + static_cast<int>(rank) * G::kRows + j * 128, row = row0 + thread;
      const uint32_t t0 = buf * 256 + lanes;
      auto drained = [&]() {  // this warp has read its part of the accumulator
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if (rank == 0)
            mbar_arrive(&s.acc_empty[buf]);
          else
            cluster_arrive_relaxed(lead + off(&s.acc_empty[buf]));
        }
      };
      if constexpr (kAct >= 0) {
        if (nh == 128) {  // 64 columns of h a warpgroup
          uint32_t g[2][16], u[2][16];
          out.begin();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t x[32], y[32], w[16];
            tmem_ld32(t0 + half * 64 + c * 32, x);
            tmem_ld32(t0 + 128 + half * 64 + c * 32, y);
            tmem_wait_ld();
            if (c == 1) drained();
            pack_row(x, g[c]);
            pack_row(y, u[c]);
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(act_value<kAct>(__uint_as_float(x[i])) * __uint_as_float(y[i]));
            pack_row(x, w);
            out.put(c, w);
          }
          const int col = n * 128 + half * 64;
          out.end(&maps.m[p.out_map], col, row0, p);
          if (p.out[1]) {
            out.begin();
            out.put(0, g[0]), out.put(1, g[1]);
            out.end(&maps.m[p.out_map + 1], col, row0, p);
          }
          if (p.out[2]) {
            out.begin();
            out.put(0, u[0]), out.put(1, u[1]);
            out.end(&maps.m[p.out_map + 2], col, row0, p);
          }
        } else {
          const int end = min(p.cols, n * nh + nh);  // a chunk may reach into the next tile's columns
          for (int c = half * 32; c < nh; c += 64) {
            uint32_t g[32], u[32], w[16];
            tmem_ld32(t0 + c, g);
            tmem_ld32(t0 + nh + c, u);
            tmem_wait_ld();
            const int col = n * nh + c;
            if (p.out[1]) pack_row(g, w), store_row(p.out[1], p.ld[1], row, col, p.rows, end, w);
            if (p.out[2]) pack_row(u, w), store_row(p.out[2], p.ld[2], row, col, p.rows, end, w);
#pragma unroll
            for (int i = 0; i < 32; ++i) g[i] = __float_as_uint(act_value<kAct>(__uint_as_float(g[i])) * __uint_as_float(u[i]));
            pack_row(g, w);
            store_row(p.out[0], p.ld[0], row, col, p.rows, end, w);
          }
          drained();
        }
      } else if (p.splits > 1) {
        // fp32, four columns of 128 rows side by side: a warp writes 512 contiguous bytes at a time
        float* const to = a.partial + (static_cast<int64_t>(p.part + tile - p.first_tile) * 2 + rank) * 256 * nh;
        for (int c = half * nh; c < (half + 1) * nh; c += 32) {
          uint32_t r[32];
          tmem_ld32(t0 + c, r);
          tmem_wait_ld();
          if (c + 32 >= (half + 1) * nh) drained();
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(to + ((c / 4 + i) * 128 + thread) * 4) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
        }
      } else {
        // nh columns a warpgroup, 64 at a time
        for (int c = 0; c < nh; c += 64) {
          out.begin();
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t r[32], w[16];
            tmem_ld32(t0 + half * nh + c + i * 32, r);
            tmem_wait_ld();
            if (i == 1 && c + 64 >= nh) drained();
            pack_row(r, w);
            out.put(i, w);
          }
          out.end(&maps.m[p.out_map], n * 2 * nh + half * nh + c, row0, p);
        }
      }
      }
    }
    if (lane == 0) tma_store_wait();
  }
  __syncwarp();
  __syncthreads();
  // After a failed wait roles of either CTA have left loads and products under way, which nobody waits for any more.
  if (*abort_flag) drain_products();
  __syncwarp();
  tc_fence_before_sync();
  cluster_sync();  // neither CTA leaves while the other may still reach its shared memory or issue products into its TMEM
  if (warp == 0) tmem_dealloc_pair(s.tmem_base, 512);
}

// The outputs of problems whose contraction is split: the parts of a tile added in their order. A block has 32 columns of a CTA's
// 128 rows.
struct SumArgs {
  Problem p[kMostProblems];
  int32_t n_problems, nh;
  const float* partial;
};
__global__ void __launch_bounds__(256) glu_sum_kernel(const __grid_constant__ SumArgs a) {
  grid_wait_predecessor();
  grid_launch_dependents();
  const int groups = a.nh / 16;  // of 32 columns
  int tile = static_cast<int>(blockIdx.x) / (2 * groups), k = 0;
  while (k + 1 < a.n_problems && tile >= a.p[k].tiles_m * a.p[k].tiles_n) tile -= a.p[k].tiles_m * a.p[k].tiles_n, ++k;
  const Problem& p = a.p[k];
  const int rest = static_cast<int>(blockIdx.x) % (2 * groups), rank = rest / groups, group = rest % groups;
  int m, n;
  tile_at<kGroupM>(p, tile * p.splits, m, n);
  const int64_t size = 256 * a.nh;
  const float* from = a.partial + (static_cast<int64_t>(p.part + tile * p.splits) * 2 + rank) * size;
  const int thread = threadIdx.x & 127, row = m * 256 + rank * 128 + thread;
  if (row >= p.rows) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = group * 32 + (2 * i + (threadIdx.x >> 7)) * 8, col = n * 2 * a.nh + c;
    if (col >= p.cols) continue;
    float4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
    const float* q = from + (c / 4 * 128 + thread) * 4;
#pragma unroll 4
    for (int part = 0; part < p.splits; ++part, q += 2 * size) {
      const float4 u = *reinterpret_cast<const float4*>(q), v = *reinterpret_cast<const float4*>(q + 512);
      x.x += u.x, x.y += u.y, x.z += u.z, x.w += u.w;
      y.x += v.x, y.y += v.y, y.z += v.z, y.w += v.w;
    }
    *reinterpret_cast<uint4*>(p.out[0] + row * p.ld[0] + col) =
        make_uint4(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w), pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
  }
}

// dg and du, 8 values a thread and access. HBM-bound: three reads and two writes of 2 bytes a value.
struct ActArgs {
  const __nv_bfloat16 *g, *u, *dh;
  __nv_bfloat16 *dg, *du;  // [rows, ff], rows on lines of 128 bytes
  int64_t ld_g, ld_u, ld_dh, ld;
  uint32_t per_row, total;  // vectors
};
template <int kAct>
__global__ void __launch_bounds__(256) glu_act_kernel(const ActArgs a) {
  grid_wait_predecessor();
  grid_launch_dependents();
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < a.total; i += gridDim.x * 256) {
    const uint32_t row = i / a.per_row, v = i - row * a.per_row;
    const uint4 g = __ldg(reinterpret_cast<const uint4*>(a.g + row * a.ld_g) + v);
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(a.u + row * a.ld_u) + v);
    const uint4 dh = __ldg(reinterpret_cast<const uint4*>(a.dh + row * a.ld_dh) + v);
    const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, uw[4] = {u.x, u.y, u.z, u.w}, hw[4] = {dh.x, dh.y, dh.z, dh.w};
    uint32_t dg[4], du[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float o[2], q[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        auto val = [&](uint32_t w) { return __uint_as_float(e ? w & 0xffff0000u : w << 16); };
        float value, slope;
        act_both<kAct>(val(gw[k]), value, slope);
        o[e] = val(hw[k]) * val(uw[k]) * slope;
        q[e] = val(hw[k]) * value;
      }
      dg[k] = pack_bf16x2(o[0], o[1]);
      du[k] = pack_bf16x2(q[0], q[1]);
    }
    reinterpret_cast<uint4*>(a.dg + row * a.ld)[v] = make_uint4(dg[0], dg[1], dg[2], dg[3]);
    reinterpret_cast<uint4*>(a.du + row * a.ld)[v] = make_uint4(du[0], du[1], du[2], du[3]);
  }
}

// ---------------------------------------------------------------- host
// A failure that a kernel recorded, per device: {code, tile, where, aux} in device memory and, for the next call to see without
// a synchronisation, in mapped host memory (as a plan has it).
__device__ int32_t g_status[4];
struct DeviceRecord {
  bool ready = false;
  StatusWord word{};
  int32_t* host = nullptr;
  int sms = 0;
};
constexpr int kMostDevices = 64;
DeviceRecord g_records[kMostDevices];
std::mutex g_mutex;

#ifdef NSP_CHECKED
std::atomic<int> g_withhold{0};
#endif
// How long a wait may take: the library's default, or where a load is withheld a thousandth of it.
void set_waits(GemmArgs& a) {
  a.wait_limit = NSP_WAIT_CYCLES_DEFAULT;
#ifdef NSP_CHECKED
  a.withhold = g_withhold.load();
  if (a.withhold) a.wait_limit = 2000000;
#endif
}

int record_of(DeviceRecord** out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= kMostDevices) return cudaGetLastError(), NSP_ERR_CUDA;
  std::lock_guard<std::mutex> lock(g_mutex);
  DeviceRecord& r = g_records[dev];
  if (!r.ready) {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // the allocation is no part of a capture that may be under way
    cudaThreadExchangeStreamCaptureMode(&mode);
    void *sym = nullptr, *host = nullptr, *mapped = nullptr;
    int major = 0;
    const bool ok = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) == cudaSuccess &&
                    cudaDeviceGetAttribute(&r.sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess &&
                    cudaGetSymbolAddress(&sym, g_status) == cudaSuccess && cudaHostAlloc(&host, 16, cudaHostAllocMapped) == cudaSuccess &&
                    cudaHostGetDevicePointer(&mapped, host, 0) == cudaSuccess;
    cudaThreadExchangeStreamCaptureMode(&mode);
    if (!ok) return cudaGetLastError(), NSP_ERR_CUDA;
    if (major != 10) return cudaFreeHost(host), NSP_ERR_UNSUPPORTED;
    r.host = static_cast<int32_t*>(host);
    r.host[0] = r.host[1] = r.host[2] = r.host[3] = 0;
    r.word = StatusWord{static_cast<int32_t*>(sym), static_cast<int32_t*>(mapped)};
    r.ready = true;
  }
  *out = &r;
  return *reinterpret_cast<volatile int32_t*>(r.host);
}

bool encode(CUtensorMap* out, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const cuuint32_t step[3] = {1, 1, 1};
  TensorMapEncoder enc = tensor_map_encoder();
  return enc && enc(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// A matrix in boxes of 64 columns
bool encode_plain(CUtensorMap* out, const void* base, int64_t cols, int64_t rows, int64_t ld, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)};
  return encode(out, base, 2, dims, strides, box);
}
// The two maps of an operand (see load_operand): boxes of `box_rows` rows and several blocks of 64 columns, and the plain matrix.
// The first one covers whole blocks alone, so that no box of it reads past the end of a row.
// The plain one is left out where no box is cut.
bool encode_operand(CUtensorMap* out, const void* base, int64_t cols, int64_t rows, int64_t ld, int box_rows, int box_cols) {
  const int blocks = box_cols / 64;
  const cuuint64_t dims[3] = {64, static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(cols < 64 ? 1 : cols / 64)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, 128};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_rows), static_cast<cuuint32_t>(blocks)};
  return (cols < box_cols || encode(out, base, 3, dims, strides, box)) && (cols % box_cols == 0 || encode_plain(out + 1, base, cols, rows, ld, box_rows));
}

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

// The order of n_long tiles of `cost` stages and n_short of `less` <= cost for that many pairs: `ahead` and `start` of the smallest
// latest end. (4,099 tokens, 2,056 x 5,512 backward: 153 tiles of 88 stages and 396 of 33; the latest pair has 429 stages where all
// tiles are dealt out one by one, 374 so, of a mean of 359.)
Schedule plan_schedule(int n_long, int cost, int n_short, int less, int pairs, int64_t* latest) {
  const int heavy = n_long % pairs, light = pairs - heavy, rounds = n_long / pairs;
  Schedule best{n_long, n_short, heavy, 0, 0};
  *latest = static_cast<int64_t>(rounds + (heavy > 0)) * cost;
  if (n_short == 0) return best;
  int64_t best_end = -1;
  const int level = heavy ? cost / less : 0;  // rounds ahead that even out what the heavy pairs have more
  for (int ahead = level > 1 ? level - 1 : 0; ahead <= level + 1; ++ahead) {
    for (int start : {0, heavy}) {
      const int64_t rest = n_short - static_cast<int64_t>(ahead) * light;  // of the rounds that all pairs take part in
      int64_t of_heavy = 0, of_light;
      if (rest <= 0) {
        of_light = (n_short + light - 1) / light;
      } else {
        const int64_t more = rest % pairs;  // pairs with one more, from `start` on
        of_heavy = rest / pairs + (more > (start == 0 ? 0 : light));
        of_light = ahead + rest / pairs + (more > (start == 0 ? heavy : 0));
      }
      const int64_t a = heavy ? static_cast<int64_t>(rounds + 1) * cost + of_heavy * less : 0;
      const int64_t b = static_cast<int64_t>(rounds) * cost + of_light * less;
      if (best_end < 0 || (a > b ? a : b) < best_end) best = Schedule{n_long, n_short, heavy, ahead, start}, best_end = a > b ? a : b;
      if (!heavy) break;
    }
    if (!heavy) break;
  }
  *latest = best_end;
  return best;
}

template <int kAct>
cudaError_t launch_gemm(const Maps& maps, const GemmArgs& a, bool tall, int pairs, cudaStream_t st) {
  static_assert(sizeof(Maps) + sizeof(GemmArgs) <= 4000, "kernel parameters");
  void (*kernel)(const Maps, const GemmArgs) = tall ? glu_gemm_kernel<kAct, true> : glu_gemm_kernel<kAct, false>;
  static std::atomic<uint64_t> allowed[2];  // by device: the kernel may use that much shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && !(allowed[tall].load(std::memory_order_relaxed) >> dev & 1)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(Smem)));
    if (e == cudaSuccess) allowed[tall].fetch_or(uint64_t{1} << dev, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return cudaGetLastError(), e;
  count_launches(1);
  return launch_chained_if(true, kernel, 2 * pairs, kThreads, sizeof(Smem), st, maps, a);
}

// Sizes of a launch's tiles.
struct Tiling {
  bool tall;
  int rows, depth, nh, pairs;  // rows of a tile, steps of a stage, columns of a CTA's part of B
  Schedule order;
  int stages(int64_t steps) const { return static_cast<int>((steps + depth - 1) / depth); }
};

// A matrix of `rows` rows: address and row stride a TMA copy can take, and rows that do not overlap
int check(const nsp_matrix_t* t, int64_t rows, int64_t cols) {
  if (!t || !t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return NSP_ERR_INVALID_ARG;
  if (t->row_stride < 0 || t->row_stride > (int64_t{1} << 31)) return NSP_ERR_INVALID_ARG;
  if (rows > 1 && (t->row_stride < cols || t->row_stride % 8)) return NSP_ERR_INVALID_ARG;
  return NSP_OK;
}
int64_t ld_of(const nsp_matrix_t* t, int64_t rows, int64_t cols) { return rows > 1 ? t->row_stride : cols; }

// The tiles that end a launch earliest. end(t, start) plans the order for t and says how many steps of the contraction the pair with
// most work has, `start` steps added for every tile. A step of a tall tile takes kTallStep of a flat one's: measured, 2 * 0.93 beside
// flat tiles with K of 16,384, and no gain with 4,096, where a tile's start, the wait for the epilogue, is a tenth of it. A step of a
// narrower flat tile takes step(nh) of a full one's: its share of the bytes, a CTA's rows of A and nh columns of B (96 tiles of 128
// columns on 74 pairs, 128 tokens, 4,096 x 12,288: 55 us, 192 of 64 columns 66; 22 tiles, 77 tokens, 1,024 x 2,816: 11.5 us, 44 of 64
// columns 8.9). `narrow`: the column counts to try. `tall_too`: enough rows for tall tiles.
constexpr int kStartFlat = 128, kStartTall = 512;
constexpr double kTallStep = 1.86;
template <typename Step, typename End>
Tiling choose_tiling(const int* narrow, int n_narrow, bool tall_too, Step step, End end) {
  Tiling best{false, 256, Geometry<false>::kDepth, 128, 0, {}};
  double best_end = static_cast<double>(end(best, kStartFlat));
  for (int i = 0; i < n_narrow; ++i) {
    Tiling t{false, 256, Geometry<false>::kDepth, narrow[i], 0, {}};
    const double e = step(narrow[i]) * end(t, kStartFlat);
    if (e < best_end) best = t, best_end = e;
  }
  if (tall_too) {
    Tiling t{true, 512, Geometry<true>::kDepth, 128, 0, {}};
    if (kTallStep * end(t, kStartTall) <= best_end) best = t;
  }
  return best;
}

// Boxes, bytes and number of the stages (see GemmArgs). a_rows: rows there are for a K-major A; mn_steps: the longest contraction over
// MN-major operands, mn: whether A is one of them in any problem.
void set_stages(GemmArgs& a, const Tiling& t, int64_t a_rows, int64_t mn_steps, bool a_kmajor, bool a_mn, bool b_mn) {
  const int full = t.rows / 2;
  a.a_rows = a_rows < full ? static_cast<int>((a_rows + 7) / 8 * 8) : full;
  a.mn_steps = mn_steps < t.depth ? static_cast<int>((mn_steps + 15) / 16 * 16) : t.depth;
  const int k_major = a.a_rows * t.depth * 2, mn = full * a.mn_steps * 2;
  a.bytes_a = a_mn && (!a_kmajor || mn > k_major) ? mn : k_major;
  a.bytes_b = a.nh * (b_mn ? a.mn_steps : t.depth) * 2;
  const int fit = static_cast<int>(kOperands) / (a.bytes_a + a.bytes_b);
  a.stages = fit < kMostStages ? fit : kMostStages;
}

int check_sizes(int64_t rows, int32_t d_model, int32_t d_ff, int32_t act) {
  if (rows < 0 || d_model < 1 || d_ff < 1 || (act != NSP_ACT_SILU && act != NSP_ACT_GELU)) return NSP_ERR_INVALID_ARG;
  if (d_model % 8 || d_ff % 8 || d_model > NSP_GLU_MAX_DIM || d_ff > NSP_GLU_MAX_DIM || rows > INT32_MAX / 2 || rows * d_ff >= int64_t{1} << 34)
    return NSP_ERR_UNSUPPORTED;
  return NSP_OK;
}

}  // namespace
}  // namespace nsp

using namespace nsp;

extern "C" int nsp_glu_fwd(const nsp_matrix_t* x, const nsp_matrix_t* w_gate, const nsp_matrix_t* w_up, const nsp_matrix_t* h,
                           const nsp_matrix_t* g, const nsp_matrix_t* u, int64_t rows, int32_t d_model, int32_t d_ff, int32_t act,
                           void* stream) {
  int rc = check_sizes(rows, d_model, d_ff, act);
  if (rc != NSP_OK || rows == 0) return rc;
  const int T = static_cast<int>(rows);
  if ((rc = check(x, rows, d_model)) || (rc = check(w_gate, d_ff, d_model)) || (rc = check(w_up, d_ff, d_model)) || (rc = check(h, rows, d_ff)) ||
      (g && (rc = check(g, rows, d_ff))) || (u && (rc = check(u, rows, d_ff))))
    return rc;
  DeviceRecord* rec = nullptr;
  if ((rc = record_of(&rec)) != NSP_OK) return rc;
  GemmArgs a = {};
  Maps maps;
  Problem& p = a.p[0];
  const int most = rec->sms / 2;
  // columns that divide d_ff evenly among one to four rounds of all pairs
  int narrow[4], n_narrow = 0;
  const int a_box = T < 128 ? T : 128;
  const int per_round = most / ceil_div(T, 256);
  for (int round = 1; round <= 4 && per_round > 0; ++round) {
    const int nh = (ceil_div(d_ff, per_round * round) + 15) / 16 * 16;  // products of a pair have a multiple of 32 columns
    if (nh < 128) narrow[n_narrow++] = nh < 32 ? 32 : nh;
  }
  const Tiling t = choose_tiling(narrow, n_narrow, T > 256, [&](int nh) { return (a_box + nh) / (a_box + 128.0); }, [&](Tiling& t, int start) {
    const int n = ceil_div(T, t.rows) * ceil_div(d_ff, t.nh);
    t.pairs = n < most ? n : most;
    int64_t latest;
    t.order = plan_schedule(n, t.stages(d_model) * t.depth + start, 0, 0, t.pairs, &latest);
    return latest;
  });
  a.nh = t.nh;
  set_stages(a, t, rows, t.depth, true, false, false);
  p.tiles_m = ceil_div(T, t.rows), p.tiles_n = ceil_div(d_ff, t.nh);
  p.segments = 1, p.depth = d_model, p.k_iters = p.per_split = t.stages(d_model), p.splits = 1;
  p.a_map[0] = 0, p.b_map[0][0] = 2, p.b_map[0][1] = 4, p.out_map = 6;
  p.rows = T, p.cols = d_ff;
  const nsp_matrix_t* outs[3] = {h, g, u};
  for (int i = 0; i < 3; ++i) {
    if (!outs[i]) continue;
    p.out[i] = static_cast<__nv_bfloat16*>(const_cast<void*>(outs[i]->data));
    p.ld[i] = ld_of(outs[i], rows, d_ff);
    if (t.nh == 128 && !encode_plain(&maps.m[p.out_map + i], outs[i]->data, d_ff, rows, p.ld[i], 128)) return NSP_ERR_CUDA;
  }
  if (!encode_operand(&maps.m[0], x->data, d_model, rows, ld_of(x, rows, d_model), a.a_rows, t.depth) ||
      !encode_operand(&maps.m[2], w_gate->data, d_model, d_ff, ld_of(w_gate, d_ff, d_model), a.nh, t.depth) ||
      !encode_operand(&maps.m[4], w_up->data, d_model, d_ff, ld_of(w_up, d_ff, d_model), a.nh, t.depth))
    return NSP_ERR_CUDA;
  a.n_problems = 1;
  a.order = t.order;
  a.status = rec->word;
  set_waits(a);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (act == NSP_ACT_SILU ? launch_gemm<kSilu>(maps, a, t.tall, t.pairs, st) : launch_gemm<kGelu>(maps, a, t.tall, t.pairs, st)) == cudaSuccess
             ? NSP_OK : NSP_ERR_CUDA;
}

namespace {
// dg and du in the workspace: rows that begin on lines of 128 bytes, so that a box of a TMA copy touches no more lines than it has
int64_t activation_ld(int32_t d_ff) { return (d_ff + 63) / 64 * 64; }
size_t activation_bytes(int64_t rows, int32_t d_ff) { return (2 * 2 * static_cast<size_t>(rows) * activation_ld(d_ff) + 255) / 256 * 256; }
// Partial tiles of split contractions: no more than kMostPartial tiles of 256 x 256 fp32
constexpr int kMostPartial = 96;
constexpr size_t kPartialBytes = static_cast<size_t>(kMostPartial) * 256 * 256 * 4;
}  // namespace

extern "C" int nsp_glu_bwd_ws_bytes(int64_t rows, int32_t d_model, int32_t d_ff, size_t* bytes) {
  if (!bytes) return NSP_ERR_INVALID_ARG;
  const int rc = check_sizes(rows, d_model, d_ff, NSP_ACT_SILU);
  if (rc != NSP_OK) return rc;
  *bytes = activation_bytes(rows, d_ff) + kPartialBytes * (rows > 0);
  return NSP_OK;
}

extern "C" int nsp_glu_bwd(const nsp_matrix_t* dh, const nsp_matrix_t* x, const nsp_matrix_t* w_gate, const nsp_matrix_t* w_up,
                           const nsp_matrix_t* g, const nsp_matrix_t* u, const nsp_matrix_t* dx, const nsp_matrix_t* dw_gate,
                           const nsp_matrix_t* dw_up, int64_t rows, int32_t d_model, int32_t d_ff, int32_t act, void* ws, size_t ws_bytes,
                           void* stream) {
  int rc = check_sizes(rows, d_model, d_ff, act);
  if (rc != NSP_OK) return rc;
  if (!dw_gate != !dw_up) return NSP_ERR_INVALID_ARG;
  const bool want_w = dw_gate != nullptr, want_x = dx != nullptr;
  if (want_w && ((rc = check(dw_gate, d_ff, d_model)) || (rc = check(dw_up, d_ff, d_model)))) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {  // sums over nothing
    if (!want_w) return NSP_OK;
    for (const nsp_matrix_t* t : {dw_gate, dw_up})
      if (cudaMemset2DAsync(const_cast<void*>(t->data), ld_of(t, d_ff, d_model) * 2, 0, static_cast<size_t>(d_model) * 2, d_ff, st) != cudaSuccess)
        return cudaGetLastError(), NSP_ERR_CUDA;
    return NSP_OK;
  }
  const int T = static_cast<int>(rows);
  if ((rc = check(dh, rows, d_ff)) || (rc = check(g, rows, d_ff)) || (rc = check(u, rows, d_ff)) || (want_w && (rc = check(x, rows, d_model))) ||
      (want_x && ((rc = check(dx, rows, d_model)) || (rc = check(w_gate, d_ff, d_model)) || (rc = check(w_up, d_ff, d_model)))))
    return rc;
  if (!want_w && !want_x) return NSP_OK;
  size_t need = 0;
  nsp_glu_bwd_ws_bytes(rows, d_model, d_ff, &need);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < need) return NSP_ERR_WORKSPACE;
  DeviceRecord* rec = nullptr;
  if ((rc = record_of(&rec)) != NSP_OK) return rc;
  ActArgs act_args = {};
  act_args.g = static_cast<const __nv_bfloat16*>(g->data), act_args.ld_g = ld_of(g, rows, d_ff);
  act_args.u = static_cast<const __nv_bfloat16*>(u->data), act_args.ld_u = ld_of(u, rows, d_ff);
  act_args.dh = static_cast<const __nv_bfloat16*>(dh->data), act_args.ld_dh = ld_of(dh, rows, d_ff);
  act_args.dg = static_cast<__nv_bfloat16*>(ws), act_args.ld = activation_ld(d_ff), act_args.du = act_args.dg + rows * act_args.ld;
  act_args.per_row = d_ff / 8, act_args.total = static_cast<uint32_t>(rows * (d_ff / 8));
  GemmArgs a = {};
  Maps maps;
  bool ok = true;
  // dg, du as [rows, d_ff]: the contraction of dx runs along their rows, that of the weights' gradients along their columns
  const int most = rec->sms / 2;
  struct Class {  // of tiles: dW or dx
    int tiles, stages, splits, per_split;
  };
  auto classes = [&](const Tiling& t, Class& w, Class& x) {
    const int tiles_n = ceil_div(d_model, 2 * t.nh);
    w = Class{want_w ? 2 * ceil_div(d_ff, t.rows) * tiles_n : 0, t.stages(T), 1, t.stages(T)};
    x = Class{want_x ? ceil_div(T, t.rows) * tiles_n : 0, 2 * t.stages(d_ff), 1, 2 * t.stages(d_ff)};
    if (t.tall) return;
    // Where a tile alone takes longer than the pairs' share of all stages, its contraction is split: into parts of that share, of four
    // stages at least, and no more of them than the workspace holds.
    const int64_t all = static_cast<int64_t>(w.tiles) * w.stages + static_cast<int64_t>(x.tiles) * x.stages;
    const int share = static_cast<int>((all + most - 1) / most), part = share < 4 ? 4 : share;
    for (Class* c : {&w, &x}) {
      if (c->tiles == 0 || 4 * c->stages <= 5 * part) continue;
      const int room = kMostPartial / 2 / c->tiles, wanted = (c->stages + part - 1) / part, n = wanted < room ? wanted : room;
      if (n < 2) continue;
      c->per_split = (c->stages + n - 1) / n;
      c->splits = (c->stages + c->per_split - 1) / c->per_split;
    }
  };
  // Half as many columns: measured, 0.65 a step (1,000 tokens, 1,024 x 2,816: 29.5 us, full tiles 32.5; 77 tokens 16.6 / 18.5)
  const int half_columns = 64;
  const Tiling t = choose_tiling(&half_columns, 1, true, [](int) { return 0.65; }, [&](Tiling& t, int start) {
    Class w, x;
    classes(t, w, x);
    const int n_w = w.tiles * w.splits, n_x = x.tiles * x.splits;
    const int c_w = w.per_split * t.depth + start, c_x = x.per_split * t.depth + start;
    t.pairs = n_w + n_x < most ? n_w + n_x : most;
    int64_t latest;
    const bool x_long = n_x > 0 && (n_w == 0 || c_x > c_w);
    t.order = x_long ? plan_schedule(n_x, c_x, n_w, c_w, t.pairs, &latest) : plan_schedule(n_w, c_w, n_x, c_x, t.pairs, &latest);
    return latest + (w.splits > 1 || x.splits > 1 ? 1024 : 0);  // one launch more
  });
  Class w, x_class;
  classes(t, w, x_class);
  a.nh = t.nh;
  // dx contracts over d_ff, its weights MN-major; where it is wanted, that is the longest contraction over MN-major operands
  set_stages(a, t, rows, want_x && (!want_w || d_ff > T) ? d_ff : T, want_x, want_w, true);
  int n_tiles = 0, n_partial = 0;
  auto add = [&](int64_t out_rows, const Class& c, const nsp_matrix_t* out, int out_map) -> Problem& {
    Problem& p = a.p[a.n_problems++];
    p.tiles_m = ceil_div(out_rows, t.rows), p.tiles_n = ceil_div(d_model, 2 * t.nh), p.first_tile = n_tiles;
    p.rows = static_cast<int32_t>(out_rows), p.cols = d_model, p.b_mn = p.b_shared = 1;
    p.splits = c.splits, p.per_split = c.per_split, p.part = n_partial;
    p.out_map = out_map, p.out[0] = static_cast<__nv_bfloat16*>(const_cast<void*>(out->data)), p.ld[0] = ld_of(out, out_rows, d_model);
    if (c.splits == 1) ok = ok && encode_plain(&maps.m[out_map], out->data, d_model, out_rows, p.ld[0], 128);
    n_tiles += p.tiles_m * p.tiles_n * c.splits;
    if (c.splits > 1) n_partial += p.tiles_m * p.tiles_n * c.splits;
    return p;
  };
  auto add_w = [&]() {
    const nsp_matrix_t* outs[2] = {dw_gate, dw_up};
    for (int i = 0; i < 2; ++i) {
      Problem& p = add(d_ff, w, outs[i], 14 + i);
      p.segments = 1, p.depth = T, p.k_iters = t.stages(T), p.a_mn = 1;
      p.a_map[0] = p.a_map[1] = 2 * i, p.b_map[0][0] = p.b_map[0][1] = p.b_map[1][0] = p.b_map[1][1] = 4;
      ok = ok && encode_operand(&maps.m[2 * i], i ? act_args.du : act_args.dg, d_ff, rows, act_args.ld, a.mn_steps, t.rows / 2);
    }
    ok = ok && encode_operand(&maps.m[4], x->data, d_model, rows, ld_of(x, rows, d_model), a.mn_steps, t.nh);
  };
  auto add_x = [&]() {
    Problem& p = add(rows, x_class, dx, 16);
    p.segments = 2, p.depth = d_ff, p.k_iters = t.stages(d_ff);
    for (int i = 0; i < 2; ++i) {
      const nsp_matrix_t* weight = i ? w_up : w_gate;
      p.a_map[i] = 6 + 2 * i, p.b_map[i][0] = p.b_map[i][1] = 10 + 2 * i;
      ok = ok && encode_operand(&maps.m[6 + 2 * i], i ? act_args.du : act_args.dg, d_ff, rows, act_args.ld, a.a_rows, t.depth) &&
           encode_operand(&maps.m[10 + 2 * i], weight->data, d_model, d_ff, ld_of(weight, d_ff, d_model), a.mn_steps, t.nh);
    }
  };
  const bool x_long = x_class.tiles > 0 && (w.tiles == 0 || x_class.per_split > w.per_split);
  if (x_long) add_x();
  if (want_w) add_w();
  if (!x_long && want_x) add_x();
  a.order = t.order;
  a.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + activation_bytes(rows, d_ff));
  if (!ok) return NSP_ERR_CUDA;
  a.status = rec->word;
  set_waits(a);
  count_launches(1);
  const int blocks = act_args.total / 256 + 1 < 148u * 8 ? static_cast<int>(act_args.total / 256 + 1) : 148 * 8;
  if (launch_chained_if(true, act == NSP_ACT_SILU ? glu_act_kernel<kSilu> : glu_act_kernel<kGelu>, blocks, 256, 0, st, act_args) != cudaSuccess)
    return NSP_ERR_CUDA;
  if (launch_gemm<-1>(maps, a, t.tall, t.pairs, st) != cudaSuccess) return NSP_ERR_CUDA;
  SumArgs sum = {};
  int n_sum = 0;
  for (int i = 0; i < a.n_problems; ++i) {
    if (a.p[i].splits == 1) continue;
    sum.p[sum.n_problems++] = a.p[i];
    n_sum += a.p[i].tiles_m * a.p[i].tiles_n;
  }
  if (n_sum == 0) return NSP_OK;
  sum.nh = a.nh, sum.partial = a.partial;
  count_launches(1);
  return launch_chained_if(true, glu_sum_kernel, n_sum * 2 * (a.nh / 16), 256, 0, st, sum) == cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
}

extern "C" int nsp_glu_status(int32_t out[4]) {
  if (!out) return NSP_ERR_INVALID_ARG;
  DeviceRecord* rec = nullptr;
  const int rc = record_of(&rec);
  if (!rec) return rc;
  if (cudaDeviceSynchronize() != cudaSuccess) return cudaGetLastError(), NSP_ERR_CUDA;
  for (int i = 0; i < 4; ++i) out[i] = reinterpret_cast<volatile int32_t*>(rec->host)[i];
  return NSP_OK;
}

#ifdef NSP_CHECKED
extern "C" int nsp_checked_withhold_glu_load(int load) {
  if (load < 0 || load > 2) return NSP_ERR_INVALID_ARG;
  g_withhold.store(load);
  return NSP_OK;
}
#endif
