// Layer norm and RMS norm over the last axis, forward and backward (non-attention work of a layer, paper Sec. 4.1.2).
//     forward   r = (mean((x - mu)^2) + eps)^(-1/2), mu = mean(x) (RMS: 0);  y = (x - mu) r w + b
//     backward  h = (x - mu) r, t = dy w:  dx = r (t - h mean(t h) - mean(t)) (RMS: without mean(t)),
//               dw = sum over the rows of dy h, db = sum of dy
// HBM-bound: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx; a row stays in registers
// between its sums and its outputs. All sums are in fp32: mu first and then the squares around it (the difference of two large
// sums would lose the variance of rows that lie far from zero).
//
// Teams. A row belongs to a team of threads, part of a warp for short rows (heads), a block for long ones; thread i has the
// vectors i, i + team, ... of 16 bytes (bf16), single elements where the rows' addresses do not allow vectors. A team walks over
// the rows with a step of all teams and loads its next row before it sums up the present one.
// The parameters' gradients stay in fp32 registers, column by column, for all rows of a team; the teams of a block are added in
// shared memory, the blocks' sums go to the workspace and a second kernel adds them in their order: the same bits in every run.
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "nsp_internal.cuh"
#include "sm100_ptx.cuh"

using nsp::grid_launch_dependents;
using nsp::grid_wait_predecessor;
using nsp::pack_bf16x2;

namespace {

struct NormRows {
  char* p;
  int64_t outer, inner;  // bytes
};

struct NormArgs {
  NormRows x, dy, y;  // y: output (dx in the backward pass)
  const void* w;
  const void* b;
  float* mean;
  float* rstd;
  float* part;  // [2][blocks][dim]: sums of a block for dw, db
  int64_t rows;
  int32_t inner, dim, w_f32, want_grads;
  float eps, inv_dim;
};

template <typename T, int V>
struct Vec {
  static constexpr int kBytes = V * static_cast<int>(sizeof(T));
  uint32_t w[kBytes >= 4 ? kBytes / 4 : 1];
  __device__ __forceinline__ void load(const char* row, int i) {
    const char* p = row + static_cast<int64_t>(i) * kBytes;
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int k = 0; k < kBytes / 16; ++k) {
        const uint4 q = *reinterpret_cast<const uint4*>(p + 16 * k);
        w[4 * k] = q.x, w[4 * k + 1] = q.y, w[4 * k + 2] = q.z, w[4 * k + 3] = q.w;
      }
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : w) v = 0;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ static void store(char* row, int i, const float (&v)[V]) {  // the one rounding, to nearest
    char* p = row + static_cast<int64_t>(i) * kBytes;
    if constexpr (sizeof(T) == 4) {
      if constexpr (V == 1) {
        *reinterpret_cast<float*>(p) = v[0];
      } else {
#pragma unroll
        for (int k = 0; k < V / 4; ++k) *reinterpret_cast<float4*>(p + 16 * k) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
      }
    } else if constexpr (V == 1) {
      *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v[0]);
    } else {
      *reinterpret_cast<uint4*>(p) =
          make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
  }
};

// V parameters from column c on (V of 8: 16-byte aligned, see the host's choice)
template <int V>
__device__ __forceinline__ void load_params(const void* base, int f32, int c, float fallback, float (&v)[V]) {
  if (!base) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = fallback;
  } else if (f32) {
    const float* p = static_cast<const float*>(base) + c;
    if constexpr (V == 1) {
      v[0] = __ldg(p);
    } else {
#pragma unroll
      for (int k = 0; k < V / 4; ++k) {
        const float4 q = __ldg(reinterpret_cast<const float4*>(p) + k);
        v[4 * k] = q.x, v[4 * k + 1] = q.y, v[4 * k + 2] = q.z, v[4 * k + 3] = q.w;
      }
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(base) + c;
    if constexpr (V == 1) {
      v[0] = __uint_as_float(static_cast<uint32_t>(__ldg(p)) << 16);
    } else {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) v[2 * k] = __uint_as_float(w[k] << 16), v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
}

// Sums over a team of kTeam lanes of a warp (kTeam <= 32), or over the block (kTeam = 0; `slot` is one of two sets of shared
// memory, taken in turn, so that one barrier a sum is enough: a set is written again only behind the other one's barrier).
template <int kTeam, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float (*slots)[N][32], int& turn) {
#pragma unroll
  for (int o = (kTeam ? kTeam : 32) / 2; o > 0; o /= 2) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  }
  if constexpr (kTeam == 0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slots[turn][k][warp] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane < warps ? slots[turn][k][lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
    turn ^= 1;
  }
}

// The rows of a team: r, r + step, ..., with (outer, inner) kept beside r without a division inside the loop.
struct RowWalk {
  int64_t r, o, step, o_step;
  int32_t i, i_step, inner;
  __device__ __forceinline__ RowWalk(int64_t first, int64_t step_, int32_t inner_) : r(first), step(step_), inner(inner_) {
    o = r / inner, i = static_cast<int32_t>(r - o * inner);
    o_step = step / inner, i_step = static_cast<int32_t>(step - o_step * inner);
  }
  __device__ __forceinline__ void next() {
    r += step, o += o_step, i += i_step;
    if (i >= inner) i -= inner, ++o;
  }
  __device__ __forceinline__ char* at(const NormRows& t) const { return t.p + o * t.outer + i * t.inner; }
};

template <typename T, int V, int NV, int kTeam, bool kLayer>
__global__ void __launch_bounds__(kTeam ? 256 : (V == 1 ? 1024 : NV == 4 ? 512 : 256)) norm_fwd_kernel(const NormArgs a) {
  __shared__ float slots[2][1][32];
  const int team = kTeam ? kTeam : blockDim.x, teams = blockDim.x / team;
  const int me = static_cast<int>(threadIdx.x) % team;
  const int n_vec = a.dim / V;
  int turn = 0;
  grid_wait_predecessor();
  grid_launch_dependents();
  RowWalk at(static_cast<int64_t>(blockIdx.x) * teams + threadIdx.x / team, static_cast<int64_t>(gridDim.x) * teams, a.inner);
  Vec<T, V> next[NV];
  auto fetch = [&]() {
    const char* row = at.at(a.x);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      next[j].zero();
      if (at.r < a.rows && me + j * team < n_vec) next[j].load(row, me + j * team);
    }
  };
  fetch();
  // All teams of a warp take the same number of steps (shuffles); rows past the end are summed up as zeros and not written.
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < a.rows; first += at.step) {
    Vec<T, V> x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j] = next[j];
    const int64_t r = at.r;
    char* out = at.at(a.y);
    at.next();
    fetch();
    float mu = 0.f;
    if (kLayer) {
      float s[1] = {0.f};
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int k = 0; k < V; ++k) s[0] += x[j].get(k);
      }
      team_sum<kTeam, 1>(s, slots, turn);
      mu = s[0] * a.inv_dim;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (me + j * team < n_vec) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float d = x[j].get(k) - mu;
          q[0] = fmaf(d, d, q[0]);
        }
      }
    }
    team_sum<kTeam, 1>(q, slots, turn);
    const float rstd = 1.f / sqrtf(q[0] * a.inv_dim + a.eps);
    if (r < a.rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int v = me + j * team;
        if (v < n_vec) {
          float w[V], b[V], y[V];
          load_params<V>(a.w, a.w_f32, v * V, 1.f, w);
          load_params<V>(a.b, a.w_f32, v * V, 0.f, b);
#pragma unroll
          for (int k = 0; k < V; ++k) y[k] = fmaf((x[j].get(k) - mu) * rstd, w[k], b[k]);
          Vec<T, V>::store(out, v, y);
        }
      }
      if (me == 0) {
        if (a.rstd) a.rstd[r] = rstd;
        if (kLayer && a.mean) a.mean[r] = mu;
      }
    }
  }
}

template <typename T, int V, int NV, int kTeam, bool kLayer>
__global__ void __launch_bounds__(kTeam ? 256 : (V == 8 && NV == 1 ? 512 : 1024)) norm_bwd_kernel(const NormArgs a) {
  __shared__ float slots[2][2][32];
  const int team = kTeam ? kTeam : blockDim.x, teams = blockDim.x / team;
  const int me = static_cast<int>(threadIdx.x) % team;
  const int n_vec = a.dim / V;
  int turn = 0;
  float dw[NV][V], db[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int k = 0; k < V; ++k) dw[j][k] = 0.f, db[j][k] = 0.f;
  }
  grid_wait_predecessor();
  grid_launch_dependents();
  RowWalk at(static_cast<int64_t>(blockIdx.x) * teams + threadIdx.x / team, static_cast<int64_t>(gridDim.x) * teams, a.inner);
  Vec<T, V> next_x[NV], next_dy[NV];
  float next_mu = 0.f, next_r = 0.f;
  auto fetch = [&]() {
    const char* row = at.at(a.x);
    const char* grad = at.at(a.dy);
    const bool here = at.r < a.rows;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      next_x[j].zero(), next_dy[j].zero();
      if (here && me + j * team < n_vec) next_x[j].load(row, me + j * team), next_dy[j].load(grad, me + j * team);
    }
    next_r = here ? a.rstd[at.r] : 0.f;
    if (kLayer) next_mu = here ? a.mean[at.r] : 0.f;
  };
  fetch();
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < a.rows; first += at.step) {
    Vec<T, V> x[NV], dy[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j] = next_x[j], dy[j] = next_dy[j];
    const float mu = next_mu, rstd = next_r;
    const int64_t r = at.r;
    char* out = at.at(a.y);
    at.next();
    fetch();
    float s[2] = {0.f, 0.f};  // t h, t
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int v = me + j * team;
      if (v < n_vec) {
        float w[V];
        load_params<V>(a.w, a.w_f32, v * V, 1.f, w);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float h = (x[j].get(k) - mu) * rstd, g = dy[j].get(k), t = g * w[k];
          s[0] = fmaf(t, h, s[0]);
          if (kLayer) s[1] += t;
          dw[j][k] = fmaf(g, h, dw[j][k]);
          db[j][k] += g;
        }
      }
    }
    team_sum<kTeam, 2>(s, slots, turn);
    const float c1 = s[0] * a.inv_dim, c2 = s[1] * a.inv_dim;
    if (r < a.rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int v = me + j * team;
        if (v < n_vec) {
          float w[V], o[V];
          load_params<V>(a.w, a.w_f32, v * V, 1.f, w);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float h = (x[j].get(k) - mu) * rstd;
            o[k] = rstd * (fmaf(dy[j].get(k), w[k], -c2) - h * c1);
          }
          Vec<T, V>::store(out, v, o);
        }
      }
    }
  }
  if (!a.want_grads) return;
  float* const part_w = a.part + static_cast<int64_t>(blockIdx.x) * a.dim;
  float* const part_b = part_w + static_cast<int64_t>(gridDim.x) * a.dim;
  if constexpr (kTeam == 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int v = me + j * team;
      if (v < n_vec) {
#pragma unroll
        for (int k = 0; k < V; ++k) part_w[v * V + k] = dw[j][k], part_b[v * V + k] = db[j][k];
      }
    }
  } else {
    // the teams of a block, added in their order
    __shared__ float sum[256 * V * NV];
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int k = 0; k < V; ++k) sum[(threadIdx.x / team) * (kTeam * V * NV) + (me + j * team) * V + k] = pass ? db[j][k] : dw[j][k];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.dim; c += blockDim.x) {
        float total = 0.f;
        for (int t = 0; t < teams; ++t) total += sum[t * (kTeam * V * NV) + c];
        (pass ? part_b : part_w)[c] = total;
      }
    }
  }
}

// dw and db (the second half of the blocks) from the sums of the blocks: 32 columns a block, eight threads a column that take
// every eighth sum.
__global__ void __launch_bounds__(256) norm_grads_kernel(const float* part, int blocks, int dim, float* dw, float* db) {
  __shared__ float sum[8][32];
  grid_wait_predecessor();
  grid_launch_dependents();
  const int half = static_cast<int>(gridDim.x) / 2, which = static_cast<int>(blockIdx.x) >= half;
  const int c = (blockIdx.x - which * half) * 32 + (threadIdx.x & 31), k = threadIdx.x >> 5;
  float* const out = which ? db : dw;
  if (!out) return;
  const float* p = part + static_cast<int64_t>(which) * blocks * dim + c;
  float total = 0.f;
  if (c < dim) {
#pragma unroll 8
    for (int i = k; i < blocks; i += 8) total += p[static_cast<int64_t>(i) * dim];
  }
  sum[k][threadIdx.x & 31] = total;
  __syncthreads();
  if (k == 0 && c < dim) {
#pragma unroll
    for (int i = 1; i < 8; ++i) total += sum[i][threadIdx.x];
    out[c] = total;
  }
}

constexpr int kSms = 148;
constexpr int kTeamBlock = 256;

// How a row is divided: elements of a vector, threads of a team, vectors of a thread, blocks an SM (of the walk).
struct Shape {
  int vec, team, per, block;
  bool whole;  // the team is the block
};
Shape shape_of(int dim, bool vectors, bool backward) {
  Shape s{vectors ? 8 : 1, 0, 1, kTeamBlock, false};
  const int n = dim / s.vec;
  if (!vectors) {
    s.per = 8;
    if (n <= 256) {
      s.team = 32;
    } else {
      if (n > 8192) s.per = 16;
      s.team = s.block = ((n + s.per - 1) / s.per + 31) / 32 * 32, s.whole = true;
    }
    return s;
  }
  if (n <= 8) s.team = 8;
  else if (n <= 16) s.team = 16;
  else if (n <= 32) s.team = 32;
  else if (n <= 64) s.team = 32, s.per = 2;
  else {
    s.whole = true;
    s.per = backward ? (n <= 512 ? 1 : 2) : (n <= 256 ? 1 : n <= 512 ? 2 : 4);
    s.team = s.block = ((n + s.per - 1) / s.per + 31) / 32 * 32;
  }
  return s;
}
int blocks_of(const Shape& s, int64_t rows) {
  const int64_t teams = s.block / s.team, need = (rows + teams - 1) / teams;
  const int64_t most = kSms * (s.block >= 1024 ? 1 : 1024 / s.block);
  return static_cast<int>(need < most ? need : most);
}

template <template <typename, int, int, int, bool> class K, typename T, bool kLayer>
void (*pick(const Shape& s))(const NormArgs) {
  if (s.vec == 1) {
    if (!s.whole) return K<T, 1, 8, 32, kLayer>::fn();
    return s.per == 8 ? K<T, 1, 8, 0, kLayer>::fn() : K<T, 1, 16, 0, kLayer>::fn();
  }
  if (!s.whole) {
    if (s.per == 2) return K<T, 8, 2, 32, kLayer>::fn();
    return s.team == 8 ? K<T, 8, 1, 8, kLayer>::fn() : s.team == 16 ? K<T, 8, 1, 16, kLayer>::fn() : K<T, 8, 1, 32, kLayer>::fn();
  }
  return s.per == 1 ? K<T, 8, 1, 0, kLayer>::fn() : s.per == 2 ? K<T, 8, 2, 0, kLayer>::fn() : K<T, 8, 4, 0, kLayer>::fn();
}
template <typename T, int V, int NV, int kTeam, bool kLayer>
struct Fwd {
  static auto fn() { return norm_fwd_kernel<T, V, NV, kTeam, kLayer>; }
};
template <typename T, int V, int NV, int kTeam, bool kLayer>
struct Bwd {
  static auto fn() { return norm_bwd_kernel<T, V, (V * NV > 16 ? 2 : NV), kTeam, kLayer>; }  // four vectors: forward only
};

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

constexpr int64_t kMostStride = int64_t{1} << 31;  // elements: with 2^31 rows at most, offsets stay inside 64 bits

// A tensor of rows: addresses and, for one that is written, rows that do not overlap. *vectors: cleared where 16-byte accesses do not fit.
int check_rows(const nsp_rows_t* t, int64_t outer, int32_t inner, int32_t dim, int size, bool written, bool* vectors, NormRows* out) {
  if (!t || !t->data || !aligned(t->data, size)) return NSP_ERR_INVALID_ARG;
  if (t->outer_stride < 0 || t->inner_stride < 0 || t->outer_stride > kMostStride || t->inner_stride > kMostStride) return NSP_ERR_INVALID_ARG;
  const int64_t o = outer > 1 ? t->outer_stride : 0, i = inner > 1 ? t->inner_stride : 0;
  if (written) {
    const bool apart = outer <= 1 ? inner <= 1 || i >= dim
                       : inner <= 1 ? o >= dim
                       : o >= i ? i >= dim && o >= (inner - 1) * i + dim
                                : o >= dim && i >= (outer - 1) * o + dim;
    if (!apart) return NSP_ERR_INVALID_ARG;
  }
  if (!aligned(t->data, 16) || o * size % 16 || i * size % 16) *vectors = false;
  *out = NormRows{static_cast<char*>(const_cast<void*>(t->data)), o * size, i * size};
  return NSP_OK;
}

int check_common(int64_t outer, int32_t inner, int32_t dim, int32_t dtype, int32_t w_dtype, int32_t kind, const void* w, const void* b) {
  if (outer < 0 || inner < 1 || dim < 1 || (dtype != NSP_BF16 && dtype != NSP_F32) || (w_dtype != NSP_BF16 && w_dtype != NSP_F32) ||
      (kind != NSP_NORM_LAYER && kind != NSP_NORM_RMS))
    return NSP_ERR_INVALID_ARG;
  if (dim > NSP_NORM_MAX_DIM || outer > INT32_MAX || outer * inner > INT32_MAX) return NSP_ERR_UNSUPPORTED;
  const size_t size = w_dtype == NSP_F32 ? 4 : 2;
  if (!aligned(w, size) || !aligned(b, size)) return NSP_ERR_INVALID_ARG;
  return NSP_OK;
}

bool same_place(const NormRows& a, const NormRows& b) { return a.p != b.p || (a.outer == b.outer && a.inner == b.inner); }

}  // namespace

extern "C" int nsp_norm_fwd(const nsp_rows_t* x, const void* weight, const void* bias, const nsp_rows_t* y, float* mean, float* rstd,
                            int64_t outer, int32_t inner, int32_t dim, int32_t dtype, int32_t w_dtype, int32_t kind, float eps,
                            void* stream) {
  int rc = check_common(outer, inner, dim, dtype, w_dtype, kind, weight, bias);
  if (rc != NSP_OK) return rc;
  if (!(eps >= 0.f) || !std::isfinite(eps) || !aligned(mean, 4) || !aligned(rstd, 4)) return NSP_ERR_INVALID_ARG;
  if (outer == 0) return NSP_OK;
  NormArgs a = {};
  const int size = dtype == NSP_F32 ? 4 : 2;
  bool vectors = dim % 8 == 0 && aligned(weight, 16) && aligned(bias, 16);
  rc = check_rows(x, outer, inner, dim, size, false, &vectors, &a.x);
  if (rc == NSP_OK) rc = check_rows(y, outer, inner, dim, size, true, &vectors, &a.y);
  if (rc != NSP_OK) return rc;
  if (!same_place(a.x, a.y)) return NSP_ERR_INVALID_ARG;
  a.w = weight, a.b = bias, a.mean = mean, a.rstd = rstd;
  a.rows = outer * inner, a.inner = inner, a.dim = dim, a.w_f32 = w_dtype == NSP_F32;
  a.eps = eps, a.inv_dim = 1.f / static_cast<float>(dim);
  const Shape s = shape_of(dim, vectors, false);
  const bool layer = kind == NSP_NORM_LAYER;
  void (*kernel)(const NormArgs) = dtype == NSP_F32 ? (layer ? pick<Fwd, float, true>(s) : pick<Fwd, float, false>(s))
                                                    : (layer ? pick<Fwd, __nv_bfloat16, true>(s) : pick<Fwd, __nv_bfloat16, false>(s));
  nsp::count_launches(1);
  return nsp::launch_chained_if(true, kernel, blocks_of(s, a.rows), s.block, 0, static_cast<cudaStream_t>(stream), a) == cudaSuccess
             ? NSP_OK : NSP_ERR_CUDA;
}

extern "C" int nsp_norm_bwd_ws_bytes(int64_t rows, int32_t dim, size_t* bytes) {
  if (!bytes || rows < 0 || dim < 1) return NSP_ERR_INVALID_ARG;
  if (dim > NSP_NORM_MAX_DIM || rows > INT32_MAX) return NSP_ERR_UNSUPPORTED;
  int most = 0;
  for (bool vectors : {false, true}) {
    const int n = blocks_of(shape_of(dim, vectors, true), rows);
    most = n > most ? n : most;
  }
  *bytes = 2 * sizeof(float) * static_cast<size_t>(most) * dim;
  return NSP_OK;
}

extern "C" int nsp_norm_bwd(const nsp_rows_t* x, const nsp_rows_t* dy, const void* weight, const float* mean, const float* rstd,
                            const nsp_rows_t* dx, float* dweight, float* dbias, int64_t outer, int32_t inner, int32_t dim, int32_t dtype,
                            int32_t w_dtype, int32_t kind, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_common(outer, inner, dim, dtype, w_dtype, kind, weight, nullptr);
  if (rc != NSP_OK) return rc;
  if (!aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return NSP_ERR_INVALID_ARG;
  const bool layer = kind == NSP_NORM_LAYER, grads = dweight || dbias;
  NormArgs a = {};
  bool vectors = dim % 8 == 0 && aligned(weight, 16);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int blocks = 0;
  a.rows = outer * inner;
  if (outer > 0) {
    if (!rstd || (layer && !mean)) return NSP_ERR_INVALID_ARG;
    const int size = dtype == NSP_F32 ? 4 : 2;
    rc = check_rows(x, outer, inner, dim, size, false, &vectors, &a.x);
    if (rc == NSP_OK) rc = check_rows(dy, outer, inner, dim, size, false, &vectors, &a.dy);
    if (rc == NSP_OK) rc = check_rows(dx, outer, inner, dim, size, true, &vectors, &a.y);
    if (rc != NSP_OK) return rc;
    if (!same_place(a.x, a.y) || !same_place(a.dy, a.y)) return NSP_ERR_INVALID_ARG;
    const Shape s = shape_of(dim, vectors, true);
    blocks = blocks_of(s, a.rows);
    if (grads && (!ws || !aligned(ws, 16) || ws_bytes < 2 * sizeof(float) * static_cast<size_t>(blocks) * dim)) return NSP_ERR_WORKSPACE;
    a.w = weight, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.part = static_cast<float*>(ws);
    a.inner = inner, a.dim = dim, a.w_f32 = w_dtype == NSP_F32, a.want_grads = grads, a.inv_dim = 1.f / static_cast<float>(dim);
    void (*kernel)(const NormArgs) = dtype == NSP_F32 ? (layer ? pick<Bwd, float, true>(s) : pick<Bwd, float, false>(s))
                                                      : (layer ? pick<Bwd, __nv_bfloat16, true>(s) : pick<Bwd, __nv_bfloat16, false>(s));
    nsp::count_launches(1);
    if (nsp::launch_chained_if(true, kernel, blocks, s.block, 0, st, a) != cudaSuccess) return NSP_ERR_CUDA;
  }
  if (!grads) return NSP_OK;
  nsp::count_launches(1);
  return nsp::launch_chained_if(true, norm_grads_kernel, 2 * ((dim + 31) / 32), 256, 0, st, static_cast<const float*>(ws), blocks, dim,
                                dweight, dbias) == cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
}
