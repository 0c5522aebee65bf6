// The gated half of a feed-forward block, forward and backward (non-attention work of a layer, paper Sec. 4.1.2), on the
// 5th-generation tensor cores.
//     forward   g = x Wg^T, u = x Wu^T, h = act(g) u, from one pass over x: the tile of g and the tile of u of the same columns are
//               one accumulator, side by side, and the activation and the product are its epilogue
//     backward  dg = dh u act'(g), du = dh act(g) (one elementwise pass, rounded to bf16: they are operands of products next);
//               dWg = dg^T x, dWu = du^T x, dx = dg Wg + du Wu, all three in one launch
// 4 T d f flop there and 8 T d f back: bound by the tensor cores from some hundred tokens on, below by the bytes of the weights.
//
// Products. A pair of CTAs (tcgen05 cta_group::2) computes tiles of 256 rows x 2 `nh` columns: each CTA loads its own 128 rows of A
// and its own nh rows of B by TMA, so that a byte of either operand is staged once for the two SMs that use it. In the forward pass
// the first CTA's part of B comes from Wg and the second one's from Wu. Operands whose contraction index is not the contiguous one
// (dg^T, du^T, x, and the weights of dx) are read MN-major by the tensor core: nothing is transposed in memory. Accumulators in
// TMEM are double-buffered: 256 columns of the next tile are filled while the epilogue drains the last one's.
#include <cmath>
#include <cstdint>
#include <mutex>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "nsp_internal.cuh"
#include "sm100_ptx.cuh"

namespace nsp {
namespace {

constexpr int kStages = 6;
constexpr uint32_t kOperand = 128 * 64 * 2;  // bytes: 128 rows (or 64 contraction steps of 2 x 64 columns) of 64 bf16
constexpr int kThreads = 384;                // producer, issuer, two idle warps, two warpgroups of epilogue
constexpr int kGroupM = 8;                   // row tiles that are walked together (see tile_at)
constexpr long long kWaitLimit = NSP_WAIT_CYCLES_DEFAULT;
constexpr int kMostMaps = 10, kMostProblems = 3;

struct Problem {
  int32_t tiles_m, tiles_n, first_tile;
  int32_t segments, k_iters;       // the contraction: `segments` pairs of operands, k_iters steps of 64 each
  int32_t a_map[2], b_map[2][2];   // [segment], [segment][rank of the CTA]
  int32_t a_mn, b_mn;              // 1: the contiguous index is the row / column one
  int32_t b_shared;                // 1: both CTAs' parts of B come from one matrix, nh columns apart
  int32_t rows, cols;              // of the output
  __nv_bfloat16* out[3];           // forward: h, g, u
  int64_t ld[3];
};

struct GemmArgs {
  Problem p[kMostProblems];
  int32_t n_problems, n_tiles, nh;
  StatusWord status;
};

struct Maps {
  CUtensorMap m[kMostMaps];
};

struct Smem {
  uint8_t a[kStages][kOperand];
  uint8_t b[kStages][kOperand];
  uint64_t full[kStages];    // in the first CTA: the bytes of both
  uint64_t empty[kStages];   // in both: the products of the stage have completed
  uint64_t acc_full[2];      // in both: an accumulator is complete
  uint64_t acc_empty[2];     // in the first CTA: 16 warps have read it
  uint32_t tmem_base;
  int32_t abort;
};
static_assert(sizeof(Smem) <= 232448, "shared memory budget (227 KB)");

enum Act : int32_t { kSilu = NSP_ACT_SILU, kGelu = NSP_ACT_GELU };

// act(x), and its slope; exp and erfc are CUDA's. The normal distribution function is erfc(-x / sqrt 2) / 2: as (1 + erf) / 2 it
// would have no correct digit left for x below -5.
__device__ __forceinline__ float normal_cdf(float x) { return 0.5f * erfcf(x * -0.70710678118654752f); }
template <int kAct>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (kAct == kSilu) return __fdividef(x, 1.f + __expf(-x));
  return x * normal_cdf(x);
}
template <int kAct>
__device__ __forceinline__ void act_both(float x, float& value, float& slope) {
  if constexpr (kAct == kSilu) {
    const float p = __fdividef(1.f, 1.f + __expf(-x));
    value = x * p;
    slope = p * (1.f + x * (1.f - p));
  } else {
    const float p = normal_cdf(x);
    value = x * p;
    slope = fmaf(x * 0.39894228040143268f, __expf(-0.5f * x * x), p);
  }
}

// The tiles of a problem: kGroupM row tiles at a time, over all column tiles, so that the tiles under way at one time share
// both their rows and their columns in L2.
__device__ __forceinline__ void tile_at(const Problem& p, int tile, int& m, int& n) {
  const int per_group = kGroupM * p.tiles_n, group = tile / per_group, rest = tile - group * per_group;
  const int first = group * kGroupM, size = min(kGroupM, p.tiles_m - first);
  n = rest / size;
  m = first + rest - n * size;
}

__device__ __forceinline__ void tma_load_2d_pair(void* smem_dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}

// 32 columns of one row
__device__ __forceinline__ void store_row(__nv_bfloat16* out, int64_t ld, int row, int col, int rows, int cols, const uint32_t (&w)[16]) {
  if (row >= rows) return;
  __nv_bfloat16* p = out + row * ld + col;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (col + 8 * i < cols) *reinterpret_cast<uint4*>(p + 8 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

__device__ __forceinline__ void pack_row(const uint32_t (&r)[32], uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
}

// kAct < 0: the accumulator is the output; otherwise the forward pass with that activation
template <int kAct>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) glu_gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ GemmArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem& s = *reinterpret_cast<Smem*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&s.full[i], 1), mbar_init(&s.empty[i], 1);
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
  auto problem_of = [&](int tile) -> const Problem& {
    int k = 0;
    while (k + 1 < a.n_problems && tile >= a.p[k + 1].first_tile) ++k;
    return a.p[k];
  };

  if (warp == 0) {
    // ================================================================ TMA producer (both CTAs, each its own operands)
    if (lane == 0) {
      uint32_t it = 0;
      for (int tile = pair; tile < a.n_tiles; tile += pairs) {
        const Problem& p = problem_of(tile);
        int m, n;
        tile_at(p, tile - p.first_tile, m, n);
        const int row = m * 256 + static_cast<int>(rank) * 128;
        const int col = p.b_shared ? n * 2 * nh + static_cast<int>(rank) * nh : n * nh;
        bool ok = true;
        for (int seg = 0; seg < p.segments && ok; ++seg) {
          const CUtensorMap* ma = &maps.m[p.a_map[seg]];
          const CUtensorMap* mb = &maps.m[p.b_map[seg][rank]];
          for (int k = 0; k < p.k_iters; ++k, ++it) {
            const uint32_t st = it % kStages, ph = (it / kStages) & 1;
            if (*abort_flag || !mbar_wait(&s.empty[st], ph ^ 1, kWaitLimit)) {
              if (!*abort_flag) report_timeout(a.status, tile, kWhereGluEmpty, k);
              raise_abort();
              ok = false;
              break;
            }
            if (rank == 0) mbar_expect_tx(&s.full[st], 2 * (kOperand + nh * 128));
            const uint32_t bar = lead + off(&s.full[st]);
            if (p.a_mn) {
              tma_load_2d_pair(s.a[st], ma, bar, row, k * 64);
              tma_load_2d_pair(s.a[st] + kOperand / 2, ma, bar, row + 64, k * 64);
            } else {
              tma_load_2d_pair(s.a[st], ma, bar, k * 64, row);
            }
            if (p.b_mn) {
              for (int c = 0; c < nh; c += 64) tma_load_2d_pair(s.b[st] + c * 128, mb, bar, col + c, k * 64);
            } else {
              tma_load_2d_pair(s.b[st], mb, bar, k * 64, col);
            }
          }
        }
        if (!ok) break;
      }
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ================================================================ issuer of the products, for both CTAs
    const bool leader = elect_one();
    const uint32_t hi = static_cast<uint32_t>(make_smem_desc_sw128(0, 16, 1024) >> 32);
    uint32_t it = 0, n_done = 0;
    bool ok = true;
    for (int tile = pair; tile < a.n_tiles && ok; tile += pairs, ++n_done) {
      const Problem& p = problem_of(tile);
      const uint32_t buf = n_done & 1, d = buf * 256;
      const uint32_t idesc = make_idesc_bf16(256, 2 * nh, p.a_mn, p.b_mn);
      // a step of 16 of the contraction: 32 bytes of a row, or 16 rows
      const uint32_t a_lbo = p.a_mn ? ((kOperand / 2) >> 4) << 16 : 1u << 16, a_step = p.a_mn ? 128 : 2;
      const uint32_t b_lbo = p.b_mn ? ((kOperand / 2) >> 4) << 16 : 1u << 16, b_step = p.b_mn ? 128 : 2;
      bool here = cluster_wait_tmem(&s.acc_empty[buf], ((n_done >> 1) & 1) ^ 1, kWaitLimit);
      if (!__all_sync(0xffffffffu, here)) {
        if (lane == 0) report_timeout(a.status, tile, kWhereGluAccEmpty, 0), raise_abort();
        break;
      }
      tc_fence_after_sync();
      const int iters = p.segments * p.k_iters;
      for (int k = 0; k < iters; ++k, ++it) {
        const uint32_t st = it % kStages, ph = (it / kStages) & 1;
        here = *abort_flag == 0 && cluster_wait(&s.full[st], ph, kWaitLimit);
        if (!__all_sync(0xffffffffu, here)) {
          if (lane == 0 && !*abort_flag) report_timeout(a.status, tile, kWhereGluFull, k);
          if (lane == 0) raise_abort();
          ok = false;
          break;
        }
        tc_fence_after_sync();
        if (leader) {
          const uint32_t a_lo = smem_desc_addr(s.a[st]) | a_lbo, b_lo = smem_desc_addr(s.b[st]) | b_lbo;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) umma2_ss_lh(d, a_lo + kk * a_step, hi, b_lo + kk * b_step, hi, idesc, (k | kk) != 0);
          umma2_commit(&s.empty[st]);
          if (k + 1 == iters) umma2_commit(&s.acc_full[buf]);
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    // ================================================================ epilogue: a warpgroup has half of the columns
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    uint32_t n_done = 0;
    for (int tile = pair; tile < a.n_tiles; tile += pairs, ++n_done) {
      const Problem& p = problem_of(tile);
      int m, n;
      tile_at(p, tile - p.first_tile, m, n);
      const uint32_t buf = n_done & 1;
      const bool here = *abort_flag == 0 && mbar_wait(&s.acc_full[buf], (n_done >> 1) & 1, kWaitLimit);
      if (!__all_sync(0xffffffffu, here)) {
        if (lane == 0 && !*abort_flag) report_timeout(a.status, tile, kWhereGluAccFull, 0);
        if (lane == 0) raise_abort();
        break;
      }
      tc_fence_after_sync();
      const int row = m * 256 + static_cast<int>(rank) * 128 + quad * 32 + lane;
      const uint32_t t0 = buf * 256 + lanes;
      if constexpr (kAct >= 0) {
        const int per = nh / 2;  // columns of h of this warpgroup
        for (int c = half * per; c < (half + 1) * per; c += 32) {
          uint32_t g[32], u[32], w[16];
          tmem_ld32(t0 + c, g);
          tmem_ld32(t0 + nh + c, u);
          tmem_wait_ld();
          const int col = n * nh + c;
          if (p.out[1]) pack_row(g, w), store_row(p.out[1], p.ld[1], row, col, p.rows, p.cols, w);
          if (p.out[2]) pack_row(u, w), store_row(p.out[2], p.ld[2], row, col, p.rows, p.cols, w);
#pragma unroll
          for (int i = 0; i < 32; ++i) g[i] = __float_as_uint(act_value<kAct>(__uint_as_float(g[i])) * __uint_as_float(u[i]));
          pack_row(g, w);
          store_row(p.out[0], p.ld[0], row, col, p.rows, p.cols, w);
        }
      } else {
        for (int c = half * nh; c < (half + 1) * nh; c += 32) {
          uint32_t r[32], w[16];
          tmem_ld32(t0 + c, r);
          tmem_wait_ld();
          pack_row(r, w);
          store_row(p.out[0], p.ld[0], row, n * 2 * nh + c, p.rows, p.cols, w);
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (rank == 0)
          mbar_arrive(&s.acc_empty[buf]);
        else
          cluster_arrive_relaxed(lead + off(&s.acc_empty[buf]));
      }
    }
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

// dg and du, 8 values a thread and access. HBM-bound: three reads and two writes of 2 bytes a value.
struct ActArgs {
  const __nv_bfloat16 *g, *u, *dh;
  __nv_bfloat16 *dg, *du;  // [rows, ff], contiguous
  int64_t ld_g, ld_u, ld_dh;
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
    reinterpret_cast<uint4*>(a.dg)[i] = make_uint4(dg[0], dg[1], dg[2], dg[3]);
    reinterpret_cast<uint4*>(a.du)[i] = make_uint4(du[0], du[1], du[2], du[3]);
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

bool encode(CUtensorMap* out, const void* base, int64_t inner, int64_t rows, int64_t ld, int box_inner, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_inner), static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t step[2] = {1, 1};
  TensorMapEncoder enc = tensor_map_encoder();
  return enc && enc(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

template <int kAct>
cudaError_t launch_gemm(const Maps& maps, const GemmArgs& a, int sms, cudaStream_t st) {
  static_assert(sizeof(Maps) + sizeof(GemmArgs) <= 4000, "kernel parameters");
  const cudaError_t e = cudaFuncSetAttribute(glu_gemm_kernel<kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(Smem)));
  if (e != cudaSuccess) return e;
  const int pairs = a.n_tiles < sms / 2 ? a.n_tiles : sms / 2;
  count_launches(1);
  return launch_chained_if(true, glu_gemm_kernel<kAct>, 2 * pairs, kThreads, sizeof(Smem), st, maps, a);
}

// A matrix of `rows` rows: address and row stride a TMA copy can take, and rows that do not overlap
int check(const nsp_matrix_t* t, int64_t rows, int64_t cols) {
  if (!t || !t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return NSP_ERR_INVALID_ARG;
  if (t->row_stride < 0 || t->row_stride > (int64_t{1} << 31)) return NSP_ERR_INVALID_ARG;
  if (rows > 1 && (t->row_stride < cols || t->row_stride % 8)) return NSP_ERR_INVALID_ARG;
  return NSP_OK;
}
int64_t ld_of(const nsp_matrix_t* t, int64_t rows, int64_t cols) { return rows > 1 ? t->row_stride : cols; }

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
  a.nh = 128;
  Problem& p = a.p[0];
  p.tiles_m = ceil_div(T, 256), p.tiles_n = ceil_div(d_ff, a.nh);
  p.segments = 1, p.k_iters = ceil_div(d_model, 64);
  p.b_map[0][0] = 1, p.b_map[0][1] = 2;
  p.rows = T, p.cols = d_ff;
  const nsp_matrix_t* outs[3] = {h, g, u};
  for (int i = 0; i < 3; ++i) {
    if (!outs[i]) continue;
    p.out[i] = static_cast<__nv_bfloat16*>(const_cast<void*>(outs[i]->data));
    p.ld[i] = ld_of(outs[i], rows, d_ff);
  }
  if (!encode(&maps.m[0], x->data, d_model, rows, ld_of(x, rows, d_model), 64, 128) ||
      !encode(&maps.m[1], w_gate->data, d_model, d_ff, ld_of(w_gate, d_ff, d_model), 64, a.nh) ||
      !encode(&maps.m[2], w_up->data, d_model, d_ff, ld_of(w_up, d_ff, d_model), 64, a.nh))
    return NSP_ERR_CUDA;
  a.n_problems = 1, a.n_tiles = p.tiles_m * p.tiles_n;
  a.status = rec->word;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (act == NSP_ACT_SILU ? launch_gemm<kSilu>(maps, a, rec->sms, st) : launch_gemm<kGelu>(maps, a, rec->sms, st)) == cudaSuccess
             ? NSP_OK : NSP_ERR_CUDA;
}

extern "C" int nsp_glu_bwd_ws_bytes(int64_t rows, int32_t d_model, int32_t d_ff, size_t* bytes) {
  if (!bytes) return NSP_ERR_INVALID_ARG;
  const int rc = check_sizes(rows, d_model, d_ff, NSP_ACT_SILU);
  if (rc != NSP_OK) return rc;
  *bytes = 2 * 2 * static_cast<size_t>(rows) * d_ff;
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
  const size_t half = 2 * static_cast<size_t>(rows) * d_ff;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < 2 * half) return NSP_ERR_WORKSPACE;
  DeviceRecord* rec = nullptr;
  if ((rc = record_of(&rec)) != NSP_OK) return rc;
  ActArgs act_args = {};
  act_args.g = static_cast<const __nv_bfloat16*>(g->data), act_args.ld_g = ld_of(g, rows, d_ff);
  act_args.u = static_cast<const __nv_bfloat16*>(u->data), act_args.ld_u = ld_of(u, rows, d_ff);
  act_args.dh = static_cast<const __nv_bfloat16*>(dh->data), act_args.ld_dh = ld_of(dh, rows, d_ff);
  act_args.dg = static_cast<__nv_bfloat16*>(ws), act_args.du = act_args.dg + rows * d_ff;
  act_args.per_row = d_ff / 8, act_args.total = static_cast<uint32_t>(rows * (d_ff / 8));
  GemmArgs a = {};
  Maps maps;
  a.nh = 128;
  bool ok = true;
  // dg, du as [rows, d_ff]: the contraction of dx runs along their rows, that of the weights' gradients along their columns
  if (want_w) {
    const nsp_matrix_t* outs[2] = {dw_gate, dw_up};
    for (int i = 0; i < 2; ++i) {
      Problem& p = a.p[a.n_problems++];
      p.tiles_m = ceil_div(d_ff, 256), p.tiles_n = ceil_div(d_model, 2 * a.nh), p.first_tile = a.n_tiles;
      p.segments = 1, p.k_iters = ceil_div(T, 64), p.a_mn = p.b_mn = p.b_shared = 1;
      p.a_map[0] = i, p.b_map[0][0] = p.b_map[0][1] = 2;
      p.rows = d_ff, p.cols = d_model;
      p.out[0] = static_cast<__nv_bfloat16*>(const_cast<void*>(outs[i]->data)), p.ld[0] = ld_of(outs[i], d_ff, d_model);
      a.n_tiles += p.tiles_m * p.tiles_n;
      ok = ok && encode(&maps.m[i], i ? act_args.du : act_args.dg, d_ff, rows, d_ff, 64, 64);
    }
    ok = ok && encode(&maps.m[2], x->data, d_model, rows, ld_of(x, rows, d_model), 64, 64);
  }
  if (want_x) {
    Problem& p = a.p[a.n_problems++];
    p.tiles_m = ceil_div(T, 256), p.tiles_n = ceil_div(d_model, 2 * a.nh), p.first_tile = a.n_tiles;
    p.segments = 2, p.k_iters = ceil_div(d_ff, 64), p.b_mn = p.b_shared = 1;
    p.rows = T, p.cols = d_model;
    p.out[0] = static_cast<__nv_bfloat16*>(const_cast<void*>(dx->data)), p.ld[0] = ld_of(dx, rows, d_model);
    a.n_tiles += p.tiles_m * p.tiles_n;
    for (int i = 0; i < 2; ++i) {
      const nsp_matrix_t* w = i ? w_up : w_gate;
      p.a_map[i] = 3 + i, p.b_map[i][0] = p.b_map[i][1] = 5 + i;
      ok = ok && encode(&maps.m[3 + i], i ? act_args.du : act_args.dg, d_ff, rows, d_ff, 64, 128) &&
           encode(&maps.m[5 + i], w->data, d_model, d_ff, ld_of(w, d_ff, d_model), 64, 64);
    }
  }
  if (!ok) return NSP_ERR_CUDA;
  a.status = rec->word;
  count_launches(1);
  const int blocks = act_args.total / 256 + 1 < 148u * 8 ? static_cast<int>(act_args.total / 256 + 1) : 148 * 8;
  if (launch_chained_if(true, act == NSP_ACT_SILU ? glu_act_kernel<kSilu> : glu_act_kernel<kGelu>, blocks, 256, 0, st, act_args) != cudaSuccess)
    return NSP_ERR_CUDA;
  return launch_gemm<-1>(maps, a, rec->sms, st) == cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
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
