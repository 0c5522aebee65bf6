// Layer norm and RMS norm over the last axis, forward and backward (non-attention work of a layer, paper Sec. 4.1.2).
//     forward   r = (mean((x - mu)^2) + eps)^(-1/2), mu = mean(x) (RMS: 0);  y = (x - mu) r w + b
//     backward  h = (x - mu) r, t = dy w:  dx = r (t - h mean(t h) - mean(t)) (RMS: without mean(t)),
//               dw = sum over the rows of dy h, db = sum of dy
// HBM-bound: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx; a row stays in registers
// between its sums and its outputs. All sums are in fp32: mu first and then the squares around it (the difference of two large
// sums would lose the variance of rows that lie far from zero). mu is the sum's quotient and is subtracted before anything is multiplied: of
// a row whose elements are all the same nothing is left but zeros, where x r - mu r or a sum times 1 / dim leave their roundings, 2^-24 |x|
// times up to 1 / sqrt(eps).
//
// Teams. A row belongs to a team of threads: some lanes of a warp, a warp or several warps; thread i of it has the vectors i,
// i + team, ... of 8 elements. In the forward pass a team takes up to four rows together, whose loads are all under way at once
// and which share the loads of the parameters (twice the bytes of a row in bf16, where they are fp32) and the barriers of their
// sums. In the backward pass a thread keeps the parameters' gradients of its columns in fp32 registers over all rows it meets,
// which bounds its columns to 16 or 32; long rows come through shared memory some rows ahead by asynchronous copies (each thread
// copies and reads its own vectors: no barrier), and a row's sums are exchanged at one barrier. The blocks'
// gradients go to the workspace and a second kernel adds them in their order: the same bits in every run.
// Rows whose addresses do not allow vectors (14-44 % of the copy rate in bf16) go element by element through kernels of their own: short ones by lanes of a warp
// (norm_*_element_kernel), long ones by a block (norm_*_odd_kernel), whose rows come through shared memory in the 16-byte pieces they
// lie in, some rows ahead. (16,384 rows of 2,051 bf16 by loads of single elements, a row ahead in registers: 102 us there, 233 back; so 75 and 110.)
#include <cmath>
#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "nsp_internal.cuh"
#include "sm100_ptx.cuh"

using nsp::grid_launch_dependents;
using nsp::grid_wait_predecessor;
using nsp::add2;
using nsp::fma2;
using nsp::mul2;
using nsp::pack_bf16x2;
using nsp::smem_u32;

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
  int32_t inner, dim, w_f32, want_grads, stages, team;  // long rows: stages of the copies, threads of a row
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

// Sums over a warp
template <int N>
__device__ __forceinline__ void warp_sum(float (&v)[N]) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  }
}
// Sums over a block (`slots`: two sets of shared memory, taken in turn, so that one barrier a sum is enough: a set is written again only
// behind the other one's barrier).
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float (*slots)[N][32], int& turn) {
  warp_sum(v);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) slots[turn][k][warp] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = lane < warps ? slots[turn][k][lane] : 0.f;
  warp_sum(v);
  turn ^= 1;
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

// The same rows of several tensors as addresses: an addition a step, and one more where a step passes the end of the inner axis.
template <int N>
struct PointerWalk {
  char* p[N];
  int64_t step[N], wrap[N], r, r_step;
  int32_t i, i_step, inner;
  __device__ __forceinline__ PointerWalk(const NormRows (&t)[N], int64_t first, int64_t step_, int32_t inner_, int64_t more)
      : r(first), r_step(step_), inner(inner_) {
    const int64_t o = r / inner, o_step = step_ / inner;
    i = static_cast<int32_t>(r - o * inner), i_step = static_cast<int32_t>(step_ - o_step * inner);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      p[k] = t[k].p + o * t[k].outer + i * t[k].inner + more;
      step[k] = o_step * t[k].outer + i_step * t[k].inner;
      wrap[k] = t[k].outer - inner * t[k].inner;
    }
  }
  __device__ __forceinline__ void next() {
    r += r_step, i += i_step;
    const bool past = i >= inner;
    if (past) i -= inner;
#pragma unroll
    for (int k = 0; k < N; ++k) p[k] += step[k] + (past ? wrap[k] : 0);
  }
};

// sum / dim: the product with the reciprocal, and what it leaves of the sum (exact in one fma) divided once more. The mean of a row whose
// elements are all the same is that element. (16,384 rows of 2,051: 80 us, with a division 84; the aligned rows' kernel loses nothing
// by the division, 131,072 x 1,024: 98 us, so 99.)
__device__ __forceinline__ float mean_of(float sum, const NormArgs& a) {
  const float m = sum * a.inv_dim, refined = fmaf(fmaf(-m, static_cast<float>(a.dim), sum), a.inv_dim, m);
  return fabsf(m) <= 3.4028234663852886e38f ? refined : m;  // what is left of an infinite sum is no number
}

// ---------------------------------------------------------------- short rows of any address
// A warp a row, up to 8 elements a lane, the next row's in registers while this one is worked on.
constexpr int kElementMost = 256;
template <typename T, bool kLayer>
__global__ void __launch_bounds__(256) norm_fwd_element_kernel(const NormArgs a) {
  constexpr int NV = kElementMost / 32, team = 32;
  const int teams = blockDim.x / team, me = static_cast<int>(threadIdx.x) % team;
  grid_wait_predecessor();
  grid_launch_dependents();
  RowWalk at(static_cast<int64_t>(blockIdx.x) * teams + threadIdx.x / team, static_cast<int64_t>(gridDim.x) * teams, a.inner);
  Vec<T, 1> next[NV];
  auto fetch = [&]() {
    const char* row = at.at(a.x);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      next[j].zero();
      if (at.r < a.rows && me + j * team < a.dim) next[j].load(row, me + j * team);
    }
  };
  fetch();
  // All teams of a warp take the same number of steps (shuffles); rows past the end are summed up as zeros and not written.
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < a.rows; first += at.step) {
    Vec<T, 1> x[NV];
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
      for (int j = 0; j < NV; ++j) s[0] += x[j].get(0);
      warp_sum(s);
      mu = mean_of(s[0], a);
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (me + j * team < a.dim) {
        const float d = x[j].get(0) - mu;
        q[0] = fmaf(d, d, q[0]);
      }
    }
    warp_sum(q);
    const float rstd = 1.f / sqrtf(q[0] * a.inv_dim + a.eps);
    if (r < a.rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int v = me + j * team;
        if (v < a.dim) {
          float w[1], b[1], y[1];
          load_params<1>(a.w, a.w_f32, v, 1.f, w);
          load_params<1>(a.b, a.w_f32, v, 0.f, b);
          y[0] = fmaf((x[j].get(0) - mu) * rstd, w[0], b[0]);
          Vec<T, 1>::store(out, v, y);
        }
      }
      if (me == 0) {
        if (a.rstd) a.rstd[r] = rstd;
        if (kLayer && a.mean) a.mean[r] = mu;
      }
    }
  }
}

template <typename T, bool kLayer>
__global__ void __launch_bounds__(256) norm_bwd_element_kernel(const NormArgs a) {
  constexpr int NV = kElementMost / 32, team = 32;
  const int teams = blockDim.x / team, me = static_cast<int>(threadIdx.x) % team;
  float dw[NV], db[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) dw[j] = db[j] = 0.f;
  grid_wait_predecessor();
  grid_launch_dependents();
  RowWalk at(static_cast<int64_t>(blockIdx.x) * teams + threadIdx.x / team, static_cast<int64_t>(gridDim.x) * teams, a.inner);
  Vec<T, 1> next_x[NV], next_dy[NV];
  float next_mu = 0.f, next_r = 0.f;
  auto fetch = [&]() {
    const char* row = at.at(a.x);
    const char* grad = at.at(a.dy);
    const bool here = at.r < a.rows;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      next_x[j].zero(), next_dy[j].zero();
      if (here && me + j * team < a.dim) next_x[j].load(row, me + j * team), next_dy[j].load(grad, me + j * team);
    }
    next_r = here ? a.rstd[at.r] : 0.f;
    if (kLayer) next_mu = here ? a.mean[at.r] : 0.f;
  };
  fetch();
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < a.rows; first += at.step) {
    Vec<T, 1> x[NV], dy[NV];
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
      if (v < a.dim) {
        float w[1];
        load_params<1>(a.w, a.w_f32, v, 1.f, w);
        const float h = (x[j].get(0) - mu) * rstd, g = dy[j].get(0), t = g * w[0];
        s[0] = fmaf(t, h, s[0]);
        if (kLayer) s[1] += t;
        dw[j] = fmaf(g, h, dw[j]);
        db[j] += g;
      }
    }
    warp_sum(s);
    const float c1 = s[0] * a.inv_dim, c2 = s[1] * a.inv_dim;
    if (r < a.rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int v = me + j * team;
        if (v < a.dim) {
          float w[1], o[1];
          load_params<1>(a.w, a.w_f32, v, 1.f, w);
          const float h = (x[j].get(0) - mu) * rstd;
          o[0] = rstd * (fmaf(dy[j].get(0), w[0], -c2) - h * c1);
          Vec<T, 1>::store(out, v, o);
        }
      }
    }
  }
  if (!a.want_grads) return;
  float* const part_w = a.part + static_cast<int64_t>(blockIdx.x) * a.dim;
  float* const part_b = part_w + static_cast<int64_t>(gridDim.x) * a.dim;
  // the teams of a block, added in their order
  __shared__ float sum[256 * NV];
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j) sum[(threadIdx.x / team) * kElementMost + me + j * team] = pass ? db[j] : dw[j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += blockDim.x) {
      float total = 0.f;
      for (int t = 0; t < teams; ++t) total += sum[t * kElementMost + c];
      (pass ? part_b : part_w)[c] = total;
    }
  }
}

// ---------------------------------------------------------------- vectors of 8 elements
// Sums of N values over kLanes lanes: halves of the values change places with halves of the lanes until a lane has one value, so
// that N values take N + 3 shuffles instead of 5 N; sum_at(k) is the lane (of its team) that ends up with value k.
template <int N, int kLanes>
__device__ __forceinline__ float lanes_sum(float (&v)[N], int lane) {
  int o = kLanes / 2;
#pragma unroll
  for (int n = N; n > 1; n /= 2, o /= 2) {
    const bool upper = lane & o;
#pragma unroll
    for (int k = 0; k < n / 2; ++k) {
      const float give = upper ? v[k] : v[k + n / 2], keep = upper ? v[k + n / 2] : v[k];
      v[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
#pragma unroll
  for (; o > 0; o /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}
template <int N, int kLanes>
__host__ __device__ constexpr int sum_at(int k) {
  int at = 0;
  for (int n = N, o = kLanes / 2; n > 1; n /= 2, o /= 2)
    if (k >= n / 2) at |= o, k -= n / 2;
  return at;
}

__device__ __forceinline__ void row_of(uint32_t r, int inner, int64_t& o, int& i) {
  o = r / static_cast<uint32_t>(inner);
  i = static_cast<int>(r - static_cast<uint32_t>(o) * inner);
}

// kLanes lanes (a warp: kWarps of them) a row, kVecs vectors a lane, kRows rows a team
constexpr int fwd_threads(int warps) { return warps > 4 ? 32 * warps : 128; }
// Blocks an SM the registers are cut to: five where four vectors a lane are under way (2,048: 50 -> 46 us for 32,768 rows); two or three of
// the longest rows, a row a block, so that some load while others store (4,096 x 16,384: 78 us with one block of two rows, 67 so); else
// the compiler's choice (512: 50 us, cut 54).
constexpr int fwd_blocks(int vecs, int warps) { return vecs == 8 && warps == 8 ? 3 : vecs != 4 ? 0 : warps <= 4 ? 5 : 2; }
template <typename T, int kLanes, int kVecs, int kWarps, int kRows, bool kLayer>
__global__ void __launch_bounds__(fwd_threads(kWarps), fwd_blocks(kVecs, kWarps)) norm_fwd_kernel(const NormArgs a) {
  constexpr int kTeam = kLanes * kWarps, kTeams = fwd_threads(kWarps) / kTeam;
  __shared__ __align__(16) float part[2][kWarps > 1 ? kTeams : 1][kRows][kWarps];
  const int lane = static_cast<int>(threadIdx.x) % kTeam, team = static_cast<int>(threadIdx.x) / kTeam;
  const int n_vec = a.dim / 8;
  grid_wait_predecessor();
  grid_launch_dependents();
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kTeams + team) * kRows;
  Vec<T, 8> x[kRows][kVecs];
  char* out[kRows];
  {
    int64_t o;
    int i;
    row_of(static_cast<uint32_t>(first), a.inner, o, i);
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const char* row = a.x.p + o * a.x.outer + i * a.x.inner;
      out[q] = a.y.p + o * a.y.outer + i * a.y.inner;
      if (++i == a.inner) i = 0, ++o;
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        x[q][j].zero();
        if (first + q < a.rows && lane + j * kTeam < n_vec) x[q][j].load(row, lane + j * kTeam);
      }
    }
  }
  // the same sums in all threads of a team
  auto team_sum = [&](float (&v)[kRows], [[maybe_unused]] int turn) {
    const float one = lanes_sum<kRows, kLanes>(v, lane % kLanes);
    if constexpr (kWarps == 1) {
#pragma unroll
      for (int q = 0; q < kRows; ++q) v[q] = __shfl_sync(0xffffffffu, one, sum_at<kRows, kLanes>(q), kLanes);
    } else {
#pragma unroll
      for (int q = 0; q < kRows; ++q)
        if (lane % 32 == sum_at<kRows, 32>(q)) part[turn][team][q][lane / 32] = one;
      __syncthreads();
#pragma unroll
      for (int q = 0; q < kRows; ++q) {
        v[q] = part[turn][team][q][0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) v[q] += part[turn][team][q][w];
      }
    }
  };
  float mu[kRows], rstd[kRows];
#pragma unroll
  for (int q = 0; q < kRows; ++q) mu[q] = 0.f;
  if (kLayer) {
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) add2(s0, s1, s0, s1, x[q][j].get(k), x[q][j].get(k + 1));
      }
      mu[q] = s0 + s1;
    }
    team_sum(mu, 0);
#pragma unroll
    for (int q = 0; q < kRows; ++q) mu[q] /= a.dim;
  }
#pragma unroll
  for (int q = 0; q < kRows; ++q) {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      if (!kLayer || lane + j * kTeam < n_vec) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          float d0 = x[q][j].get(k), d1 = x[q][j].get(k + 1);
          if (kLayer) add2(d0, d1, d0, d1, -mu[q], -mu[q]);
          fma2(s0, s1, d0, d1, d0, d1, s0, s1);
        }
      }
    }
    rstd[q] = s0 + s1;
  }
  team_sum(rstd, 1);
#pragma unroll
  for (int q = 0; q < kRows; ++q) {
    rstd[q] = 1.f / sqrtf(rstd[q] * a.inv_dim + a.eps);
    if (lane == 0 && first + q < a.rows) {
      if (a.rstd) a.rstd[first + q] = rstd[q];
      if (kLayer && a.mean) a.mean[first + q] = mu[q];
    }
  }
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    const int v = lane + j * kTeam;
    if (v < n_vec) {
      float w[8], b[8];
      load_params<8>(a.w, a.w_f32, v * 8, 1.f, w);
      load_params<8>(a.b, a.w_f32, v * 8, 0.f, b);
#pragma unroll
      for (int q = 0; q < kRows; ++q) {
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          float d0 = x[q][j].get(k), d1 = x[q][j].get(k + 1);
          if (kLayer) add2(d0, d1, d0, d1, -mu[q], -mu[q]);
          mul2(d0, d1, d0, d1, rstd[q], rstd[q]);
          fma2(y[k], y[k + 1], d0, d1, w[k], w[k + 1], b[k], b[k + 1]);
        }
        if (first + q < a.rows) Vec<T, 8>::store(out[q], v, y);
      }
    }
  }
}

// What a thread does with a vector of a row: the sums of t h and t and the parameters' gradients, and dx. A row's constants:
//     h = (x - mu) r;   dx = (t - c2 - h c1) r,   c1 = mean(t h), c2 = mean(t)
// in that order: x r - mu r and t r - (x - mu) (r^2 c1) would save a pair of elements one and two of its instructions (layer norm, 32,768 x
// 4,096: 147.5 us with both, 149.5 with the second, 151.5 so), but leave the rounding of mu r, and r^2 leaves fp32 where the rows are of order
// 10^-19 and eps is 0.
enum : int { kRms = 0, kRmsBias = 1, kLayerBias = 2 };  // whether mean(t) is subtracted and db is summed up
// Pairs of fp32 in one 64-bit register, as the packed instructions take them.
struct F2 {
  uint64_t v;
  __device__ __forceinline__ static F2 of(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
  }
  __device__ __forceinline__ float lo() const { return __uint_as_float(static_cast<uint32_t>(v)); }
  __device__ __forceinline__ float hi() const { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
  __device__ __forceinline__ float sum() const { return lo() + hi(); }
};
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

template <typename T, int kKind>
struct BwdVec {
  struct Params {  // of the 8 columns of a vector
    F2 v[4];
    __device__ __forceinline__ void zero() {
#pragma unroll
      for (F2& x : v) x.v = 0;
    }
    __device__ __forceinline__ void load(const NormArgs& a, int c) {
      float w[8];
      load_params<8>(a.w, a.w_f32, c, 1.f, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = F2::of(w[2 * k], w[2 * k + 1]);
    }
  };
  __device__ __forceinline__ static F2 pair(const Vec<T, 8>& x, int k) { return F2::of(x.get(2 * k), x.get(2 * k + 1)); }
  __device__ __forceinline__ static void sums(const Vec<T, 8>& x, const Vec<T, 8>& dy, const Params& w, F2 r, F2 minus_mu, F2& s, F2& c, Params& dw,
                                              Params& db) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const F2 g = pair(dy, k), u = pair(x, k);
      const F2 gh = mul(mul(kKind == kLayerBias ? add(u, minus_mu) : u, r), g);
      s = fma(w.v[k], gh, s);
      dw.v[k] = add(dw.v[k], gh);
      if (kKind == kLayerBias) c = fma(w.v[k], g, c);
      if (kKind != kRms) db.v[k] = add(db.v[k], g);
    }
  }
  __device__ __forceinline__ static void grad(const Vec<T, 8>& x, const Vec<T, 8>& dy, const Params& w, F2 r, F2 minus_mu, F2 minus_c1, F2 minus_c2, char* out,
                                              int v, bool here = true) {
    float o[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const F2 u = pair(x, k);
      const F2 h = mul(kKind == kLayerBias ? add(u, minus_mu) : u, r), g = pair(dy, k);
      const F2 d = mul(fma(h, minus_c1, kKind == kLayerBias ? fma(g, w.v[k], minus_c2) : mul(g, w.v[k])), r);
      o[2 * k] = d.lo(), o[2 * k + 1] = d.hi();
    }
    if (here) Vec<T, 8>::store(out, v, o);
  }
};
__device__ __forceinline__ F2 both(float x) { return F2::of(x, x); }

// Short rows: kLanes lanes of a warp a row, kRows rows at a time
template <typename T, int kLanes, int kVecs, int kRows, int kKind>
__global__ void __launch_bounds__(256) norm_bwd_short_kernel(const NormArgs a) {
  constexpr int kTeams = 256 / kLanes, kSums = kRows * (kKind == kLayerBias ? 2 : 1);
  const int lane = static_cast<int>(threadIdx.x) % kLanes, team = static_cast<int>(threadIdx.x) / kLanes;
  const int n_vec = a.dim / 8;
  using B = BwdVec<T, kKind>;
  typename B::Params dw[kVecs], db[kVecs], w[kVecs];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) dw[j].zero(), db[j].zero(), w[j].zero();
  grid_wait_predecessor();
  grid_launch_dependents();
#pragma unroll
  for (int j = 0; j < kVecs; ++j)
    if (lane + j * kLanes < n_vec) w[j].load(a, (lane + j * kLanes) * 8);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kTeams * kRows;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kTeams * kRows; base < a.rows; base += step) {
    Vec<T, 8> x[kRows][kVecs], dy[kRows][kVecs];
    float r[kRows], minus_mu[kRows];
    char* out[kRows];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const int64_t row = base + q * kTeams + team;
      const bool here = row < a.rows;
      int64_t o;
      int i;
      row_of(static_cast<uint32_t>(row), a.inner, o, i);
      const char *px = a.x.p + o * a.x.outer + i * a.x.inner, *pg = a.dy.p + o * a.dy.outer + i * a.dy.inner;
      out[q] = here ? a.y.p + o * a.y.outer + i * a.y.inner : nullptr;
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        x[q][j].zero(), dy[q][j].zero();
        if (here && lane + j * kLanes < n_vec) x[q][j].load(px, lane + j * kLanes), dy[q][j].load(pg, lane + j * kLanes);
      }
      r[q] = here ? a.rstd[row] : 0.f;
      minus_mu[q] = kKind == kLayerBias && here ? -a.mean[row] : 0.f;
    }
    float sum[kSums];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      F2 s{0}, c{0};
#pragma unroll
      for (int j = 0; j < kVecs; ++j)
        if (lane + j * kLanes < n_vec) B::sums(x[q][j], dy[q][j], w[j], both(r[q]), both(minus_mu[q]), s, c, dw[j], db[j]);
      sum[q] = s.sum();
      if (kKind == kLayerBias) sum[kRows + q] = c.sum();
    }
    const float mine = lanes_sum<kSums, kLanes>(sum, lane) * a.inv_dim;
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const float c1 = __shfl_sync(0xffffffffu, mine, sum_at<kSums, kLanes>(q), kLanes);
      const float c2 = kKind == kLayerBias ? __shfl_sync(0xffffffffu, mine, sum_at<kSums, kLanes>(kRows + q), kLanes) : 0.f;
      if (out[q]) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
          if (lane + j * kLanes < n_vec)
            B::grad(x[q][j], dy[q][j], w[j], both(r[q]), both(minus_mu[q]), both(-c1), both(-c2), out[q], lane + j * kLanes);
      }
    }
  }
  if (!a.want_grads) return;
  // the teams of a block, added in their order
  __shared__ float sum[kTeams][kLanes * kVecs * 8 + 1];
  float* const part_w = a.part + static_cast<int64_t>(blockIdx.x) * a.dim;
  float* const part_b = part_w + static_cast<int64_t>(gridDim.x) * a.dim;
#pragma unroll
  for (int pass = 0; pass < (kKind == kRms ? 1 : 2); ++pass) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const F2 v = pass ? db[j].v[k] : dw[j].v[k];
        sum[team][(lane + j * kLanes) * 8 + 2 * k] = v.lo(), sum[team][(lane + j * kLanes) * 8 + 2 * k + 1] = v.hi();
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += 256) {
      float total = 0.f;
#pragma unroll 8
      for (int t = 0; t < kTeams; ++t) total += sum[t][c];
      (pass ? part_b : part_w)[c] = total;
    }
  }
}

// Long rows: several warps a row, kVecs vectors a thread, a.stages rows ahead. A block has one or more teams, which go on together (one
// barrier a row). One row at a time: two at one barrier take more registers than two blocks an SM have (32,768 x 4,096: 141 us, with
// two rows 276, and 512 threads of one vector 298). Rows of more than 8,192 elements take four vectors a thread: halves of a row in the CTAs
// of a cluster, its barrier hidden behind the next row's sums, gain with two sums a row and lose with one (4,096 x 16,384: layer norm 143 us,
// halves 123; RMS 110 and 111; 4,096 x 12,288 RMS 96 and 104; 8,192 x 8,320 193 and 205). The faster form for long layer norms is left for a
// kernel of its own. These figures, and those in the kernel, are of the order of products that BwdVec names as the faster one: 2-3 % are to
// be added for layer norm.
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, uint32_t bytes) {  // 16, or none: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void wait_oldest(int stages) {  // of that many groups of copies under way
  if (stages >= 3)
    asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (stages == 2)
    asm volatile("cp.async.wait_group 1;" ::: "memory");
  else
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}
template <typename T, int kThreads, int kVecs, int kKind>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) norm_bwd_long_kernel(const NormArgs a) {
  constexpr int kParts = kKind == kLayerBias ? 2 : 1, kVecBytes = 8 * static_cast<int>(sizeof(T));
  constexpr uint32_t kVecRow = kThreads * kVecBytes, kRowBytes = kVecRow * kVecs, kStageBytes = 2 * kRowBytes;
  extern __shared__ __align__(16) char ring[];  // [stages][x, dy][kVecs][threads] vectors; then the teams' gradients
  __shared__ __align__(16) float part[2][kParts][kThreads / 32];
  const int team_threads = a.team, teams = kThreads / team_threads;  // the threads behind the last team have no vectors
  const int team = static_cast<int>(threadIdx.x) / team_threads, tid = static_cast<int>(threadIdx.x) - team * team_threads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team_warps = team_threads >> 5;
  const int n_vec = team < teams ? a.dim / 8 : 0, stages = a.stages;
  // Weights and the row stay in registers between the sums and dx; with more than two vectors a thread there is no room for them: the weights
  // are loaded again, and the row is read again from its stage, which is then filled anew behind that.
  constexpr int kHeld = kVecs > 2 ? 0 : kVecs;
  using B = BwdVec<T, kKind>;
  typename B::Params dw[kVecs], db[kVecs], held[kHeld ? kHeld : 1];
  bool on[kVecs];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    on[j] = tid + j * team_threads < n_vec;
    dw[j].zero(), db[j].zero();
  }
  grid_wait_predecessor();
  grid_launch_dependents();
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    held[j].zero();
    if (on[j]) held[j].load(a, (tid + j * team_threads) * 8);
  }
  auto weights = [&](int j) -> typename B::Params {
    if constexpr (kHeld > 0) {
      return held[j];
    } else {
      typename B::Params w;
      w.zero();
      if (on[j]) w.load(a, (tid + j * team_threads) * 8);
      return w;
    }
  };
  // With three vectors a thread, a warp leaves out those that none of its lanes has: a row of 8,320 elements takes little more than two (8,192
  // rows: 156 us, with four vectors of 288 threads 193; 4,096 x 12,288 105 and 125). With four the branches cost more (4,096 x 16,384: 143 us, 153 with them).
  auto idle = [&](int j) { return kVecs == 3 && (tid & ~31) + j * team_threads >= n_vec; };
  const uint32_t mine = smem_u32(ring) + threadIdx.x * kVecBytes;
  const int64_t step = static_cast<int64_t>(gridDim.x) * teams;
  const int64_t start = static_cast<int64_t>(blockIdx.x) * teams + team;
  const int64_t thread_at = static_cast<int64_t>(tid) * kVecBytes;
  const uint32_t team_at = static_cast<uint32_t>(team_threads) * kVecBytes;
  const NormRows in_rows[2] = {a.x, a.dy}, out_rows[1] = {a.y};
  PointerWalk<2> in(in_rows, start, step, a.inner, thread_at);
  PointerWalk<1> out(out_rows, start, step, a.inner, 0);
  // The copies of the next row of the walk, one group; zeros for vectors and rows that do not exist, which then add nothing
  auto fetch = [&](int stage) {
    const uint32_t to = mine + stage * kStageBytes;
    const bool here = in.r < a.rows;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      if (idle(j)) continue;
      const uint32_t bytes = here && on[j] ? 16 : 0;
#pragma unroll
      for (int e = 0; e < kVecBytes; e += 16) {
        copy_async16(to + j * kVecRow + e, in.p[0] + j * team_at + e, bytes);
        copy_async16(to + kRowBytes + j * kVecRow + e, in.p[1] + j * team_at + e, bytes);
      }
    }
    in.next();
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < stages; ++i) fetch(i);
  float next_r, next_mu;
  auto statistics = [&](int64_t row) {
    next_r = row < a.rows ? __ldg(a.rstd + row) : 0.f;
    next_mu = kKind == kLayerBias && row < a.rows ? __ldg(a.mean + row) : 0.f;
  };
  statistics(start);
  int turn = 0, stage = 0;
  const float inv_dim = a.inv_dim;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * teams; base < a.rows; base += step, turn ^= 1) {
    const float r = next_r, minus_mu = -next_mu;
    wait_oldest(stages);
    const char* const from = ring + stage * kStageBytes + threadIdx.x * kVecBytes;
    Vec<T, 8> x[kVecs], dy[kVecs];
    auto read = [&](int j) { x[j].load(from + j * kVecRow, 0), dy[j].load(from + kRowBytes + j * kVecRow, 0); };
    F2 s{0}, c{0};
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      if (idle(j)) continue;
      read(j);
      // (a vector that does not exist is centred by a factor of 0, or its zeros would be 0 - mu, times r perhaps not finite)
      B::sums(x[j], dy[j], weights(j), both(kKind == kLayerBias && !on[j] ? 0.f : r), both(minus_mu), s, c, dw[j], db[j]);
    }
    float sum[kParts];
    sum[0] = s.sum();
    if constexpr (kKind == kLayerBias) sum[1] = c.sum();
    const int now = stage;
    if (++stage == stages) stage = 0;
    if (kHeld) fetch(now);  // over what this thread has just read
    statistics(out.r + step);
    const float one = lanes_sum<kParts, 32>(sum, lane);
#pragma unroll
    for (int k = 0; k < kParts; ++k)
      if (lane == sum_at<kParts, 32>(k)) part[turn][k][warp] = one;
    __syncthreads();  // the other set is written behind the next barrier but one at the earliest
    // The warps' sums, a value in every 8 lanes (or 16, where a team has more than 8 warps), in one order for all threads
    float total[kParts];
    {
      constexpr int kWide = kThreads > 256 ? 16 : 8;
      const int w = lane % kWide, k = lane / kWide, first_warp = min(team, teams - 1) * team_warps;
      float v = k < kParts && w < team_warps ? part[turn][k][first_warp + w] : 0.f;
#pragma unroll
      for (int o = kWide / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
      v *= inv_dim;
#pragma unroll
      for (int i = 0; i < kParts; ++i) total[i] = __shfl_sync(0xffffffffu, v, i * kWide);
    }
    const float c1 = total[0], c2 = kKind == kLayerBias ? total[kParts - 1] : 0.f;
    const bool here = out.r < a.rows;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      if (idle(j)) continue;
      if (!kHeld) read(j);
      B::grad(x[j], dy[j], weights(j), both(r), both(minus_mu), both(-c1), both(-c2), out.p[0], tid + j * team_threads, here && on[j]);
    }
    if (!kHeld) fetch(now);
    out.next();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (!a.want_grads) return;
  float* const part_w = a.part + static_cast<int64_t>(blockIdx.x) * a.dim;
  float* const part_b = part_w + static_cast<int64_t>(gridDim.x) * a.dim;
  // the teams of a block, added in their order
  float* const sums = reinterpret_cast<float*>(ring);  // [teams][vectors of a team][8]
  const int team_floats = team_threads * kVecs * 8;
#pragma unroll
  for (int pass = 0; pass < (kKind == kRms ? 1 : 2); ++pass) {
    float* const to = pass ? part_b : part_w;
    if (teams > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const F2 v = pass ? db[j].v[k] : dw[j].v[k];
          if (on[j]) *reinterpret_cast<F2*>(sums + team * team_floats + (tid + j * team_threads) * 8 + 2 * k) = v;
        }
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.dim; c += kThreads) {
        float t = sums[c];
        for (int i = 1; i < teams; ++i) t += sums[i * team_floats + c];
        to[c] = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        if (on[j]) {
          float* const at = to + (tid + j * team_threads) * 8;
#pragma unroll
          for (int k = 0; k < 4; ++k) *reinterpret_cast<F2*>(at + 2 * k) = pass ? db[j].v[k] : dw[j].v[k];
        }
      }
    }
  }
}

// ---------------------------------------------------------------- long rows of any address
// A row of `bytes` bytes at `row` into shared memory, in the 16-byte pieces that it lies in: the first and the last piece may hold
// neighbours' bytes, which nobody reads. Nothing is read behind the row's end, nor in front of `first`, the tensor's first element (such
// a piece goes element by element). Element c is at offset `row` modulo 16 plus c elements.
template <typename T>
__device__ __forceinline__ void stage_row(char* to, const char* row, int bytes, const char* first) {
  const char* const begin = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t{15});
  const int shift = static_cast<int>(row - begin), pieces = (shift + bytes + 15) / 16;
  for (int i = threadIdx.x; i < pieces; i += blockDim.x) {
    const int at = 16 * i, end = min(at + 16, shift + bytes);
    if (begin + at >= first) {
      copy_async16(smem_u32(to + at), begin + at, static_cast<uint32_t>(end - at));
    } else {
      for (int b = max(at, shift); b < end; b += static_cast<int>(sizeof(T))) *reinterpret_cast<T*>(to + b) = *reinterpret_cast<const T*>(begin + b);
    }
  }
}
template <typename T>
__device__ __forceinline__ float element(const char* p) {
  if constexpr (sizeof(T) == 4) return *reinterpret_cast<const float*>(p);
  return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
}
template <typename T>
__device__ __forceinline__ void put_element(char* p, float v) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float*>(p) = v;
  else *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
}
__host__ __device__ constexpr int odd_row_bytes(int bytes) { return (bytes + 15) / 16 * 16 + 16; }

// What a thread of these kernels has of a row: the elements tid, tid + threads, ...; the parameters of its columns stay in registers.
template <typename T, int kPer>
struct Columns {
  int first, step, n;  // bytes; elements there are
  __device__ __forceinline__ Columns(int dim) {
    const int threads = blockDim.x, tid = threadIdx.x;
    first = tid * static_cast<int>(sizeof(T)), step = threads * static_cast<int>(sizeof(T));
    n = tid < dim ? (dim - tid + threads - 1) / threads : 0;
  }
  __device__ __forceinline__ void params(const void* base, int f32, float fallback, float (&v)[kPer]) const {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      float x[1] = {0.f};
      if (j < n) load_params<1>(base, f32, threadIdx.x + j * blockDim.x, fallback, x);
      v[j] = x[0];
    }
  }
};

// A block a row, kPer elements a thread, up to kThreads threads
template <typename T, int kThreads, int kPer, bool kLayer>
__global__ void __launch_bounds__(kThreads, kPer == 8 ? 2 : 1) norm_fwd_odd_kernel(const NormArgs a) {
  extern __shared__ __align__(16) char ring[];
  __shared__ float slots[2][1][32];
  const int bytes = a.dim * static_cast<int>(sizeof(T)), row_bytes = odd_row_bytes(bytes), stages = a.stages;
  const Columns<T, kPer> mine(a.dim);
  int turn = 0, stage = 0;
  grid_wait_predecessor();
  grid_launch_dependents();
  float w[kPer], b[kPer];
  mine.params(a.w, a.w_f32, 1.f, w);
  mine.params(a.b, a.w_f32, 0.f, b);
  const NormRows rows[2] = {a.x, a.y};
  PointerWalk<2> in(rows, blockIdx.x, gridDim.x, a.inner, 0), at = in;
  auto fetch = [&](int to) {
    if (in.r < a.rows) stage_row<T>(ring + to * row_bytes, in.p[0], bytes, a.x.p);
    in.next();
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < stages; ++i) fetch(i);
  for (; at.r < a.rows; at.next()) {
    wait_oldest(stages);
    __syncthreads();  // the pieces of all threads are there
    const char* from = ring + stage * row_bytes + (reinterpret_cast<uintptr_t>(at.p[0]) & 15) + mine.first;
    float x[kPer], s[1] = {0.f}, mu = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j, from += mine.step) {
      x[j] = j < mine.n ? element<T>(from) : 0.f;
      s[0] += x[j];
    }
    if (kLayer) {
      block_sum(s, slots, turn);
      mu = mean_of(s[0], a);
    }
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const float d = x[j] - mu;
      if (j < mine.n) s[0] = fmaf(d, d, s[0]);
    }
    block_sum(s, slots, turn);
    fetch(stage);  // behind a barrier: everybody has read the row
    if (++stage == stages) stage = 0;
    const float rstd = 1.f / sqrtf(s[0] * a.inv_dim + a.eps);
    char* out = at.p[1] + mine.first;
#pragma unroll
    for (int j = 0; j < kPer; ++j, out += mine.step)
      if (j < mine.n) put_element<T>(out, fmaf((x[j] - mu) * rstd, w[j], b[j]));
    if (threadIdx.x == 0) {
      if (a.rstd) a.rstd[at.r] = rstd;
      if (kLayer && a.mean) a.mean[at.r] = mu;
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int kThreads, int kPer, bool kLayer>
__global__ void __launch_bounds__(kThreads, 1) norm_bwd_odd_kernel(const NormArgs a) {
  extern __shared__ __align__(16) char ring[];  // [stages][x, dy]
  __shared__ float slots[2][2][32];
  const int bytes = a.dim * static_cast<int>(sizeof(T)), row_bytes = odd_row_bytes(bytes), stages = a.stages;
  const Columns<T, kPer> mine(a.dim);
  int turn = 0, stage = 0;
  float w[kPer], dw[kPer], db[kPer];
  grid_wait_predecessor();
  grid_launch_dependents();
  mine.params(a.w, a.w_f32, 1.f, w);
#pragma unroll
  for (int j = 0; j < kPer; ++j) dw[j] = 0.f, db[j] = 0.f;
  RowWalk in(blockIdx.x, gridDim.x, a.inner), at = in;
  auto fetch = [&](int to) {
    if (in.r < a.rows) {
      stage_row<T>(ring + 2 * to * row_bytes, in.at(a.x), bytes, a.x.p);
      stage_row<T>(ring + (2 * to + 1) * row_bytes, in.at(a.dy), bytes, a.dy.p);
    }
    in.next();
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < stages; ++i) fetch(i);
  for (; at.r < a.rows; at.next()) {
    const float rstd = __ldg(a.rstd + at.r), mu = kLayer ? __ldg(a.mean + at.r) : 0.f;
    wait_oldest(stages);
    __syncthreads();  // the pieces of all threads are there
    const char* from = ring + 2 * stage * row_bytes + (reinterpret_cast<uintptr_t>(at.at(a.x)) & 15) + mine.first;
    const char* grad = ring + (2 * stage + 1) * row_bytes + (reinterpret_cast<uintptr_t>(at.at(a.dy)) & 15) + mine.first;
    float h[kPer], t[kPer], s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kPer; ++j, from += mine.step, grad += mine.step) {
      // (a branch: with the arithmetic done on zeros as well the 2,051-wide rows took 174 us instead of 110)
      if (static_cast<int>(threadIdx.x) + j * static_cast<int>(blockDim.x) >= a.dim) {
        h[j] = t[j] = 0.f;
        continue;
      }
      const float g = element<T>(grad);
      h[j] = (element<T>(from) - mu) * rstd;
      t[j] = g * w[j];
      s[0] = fmaf(t[j], h[j], s[0]);
      if (kLayer) s[1] += t[j];
      dw[j] = fmaf(g, h[j], dw[j]);
      db[j] += g;
    }
    block_sum(s, slots, turn);
    fetch(stage);  // behind a barrier: everybody has read the row
    if (++stage == stages) stage = 0;
    const float c1 = s[0] * a.inv_dim, c2 = s[1] * a.inv_dim;
    char* out = at.at(a.y) + mine.first;
#pragma unroll
    for (int j = 0; j < kPer; ++j, out += mine.step)
      if (j < mine.n) put_element<T>(out, rstd * (t[j] - c2 - h[j] * c1));
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (!a.want_grads) return;
  float* part_w = a.part + static_cast<int64_t>(blockIdx.x) * a.dim + threadIdx.x;
  float* part_b = part_w + static_cast<int64_t>(gridDim.x) * a.dim;
#pragma unroll
  for (int j = 0; j < kPer; ++j, part_w += blockDim.x, part_b += blockDim.x)
    if (j < mine.n) *part_w = dw[j], *part_b = db[j];
}

// dw and db (the second half of the blocks) from the sums of the blocks: 32 columns a block, a sum in turn for every warp. 32 warps where
// two blocks an SM have left theirs, 16 for fewer (148 sums of 16,384 columns: 4 us less than 32), no more than there are sums (one row of
// 16,384: 16.9 -> 15.0 us both kernels).
__global__ void __launch_bounds__(1024) norm_grads_kernel(const float* part, int blocks, int dim, float* dw, float* db) {
  __shared__ float sum[32][33];
  grid_wait_predecessor();
  grid_launch_dependents();
  const int half = static_cast<int>(gridDim.x) / 2, which = static_cast<int>(blockIdx.x) >= half;
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, warps = blockDim.x >> 5, c = (blockIdx.x - which * half) * 32 + lane;
  float* const out = which ? db : dw;
  if (!out) return;
  const float* p = part + static_cast<int64_t>(which) * blocks * dim + c;
  float total = 0.f;
  if (c < dim) {
#pragma unroll 8
    for (int i = k; i < blocks; i += warps) total += p[static_cast<int64_t>(i) * dim];
  }
  if (warps > 1) {
    sum[k][lane] = total;
    __syncthreads();
    if (k > 0) return;
    total = 0.f;
    for (int i = 0; i < warps; ++i) total += sum[i][lane];
  }
  if (c < dim) out[c] = total;
}

constexpr int kSms = 148;
constexpr int kMostShared = 227 * 1024;
constexpr int kStaticShared = 1024;  // no less than the kernels with dynamic shared memory have of their own

// A launch: which kernel, blocks and threads; shared memory, stages and threads of a row of the long rows' kernel.
struct Launch {
  void (*kernel)(const NormArgs) = nullptr;
  int64_t blocks = 0;
  int threads = 0, shared = 0, stages = 0, team = 0;
};

int round32(int n) { return (n + 31) / 32 * 32; }

// Rows whose addresses allow no vectors: up to 8 elements a lane of a warp, or up to 16 a thread of a block.
template <typename T, bool kLayer>
Launch element_launch(int dim, int64_t rows, bool backward) {
  Launch l;
  if (dim <= kElementMost) {
    l.kernel = backward ? norm_bwd_element_kernel<T, kLayer> : norm_fwd_element_kernel<T, kLayer>;
    l.threads = 256;
    const int64_t need = (rows + 7) / 8, most = kSms * 4;
    l.blocks = need < most ? need : most;
    return l;
  }
  const int per = dim <= 4096 ? 8 : 16;
  if (dim <= 4096) l.kernel = backward ? norm_bwd_odd_kernel<T, 512, 8, kLayer> : norm_fwd_odd_kernel<T, 512, 8, kLayer>;
  else if (dim <= 8192) l.kernel = backward ? norm_bwd_odd_kernel<T, 512, 16, kLayer> : norm_fwd_odd_kernel<T, 512, 16, kLayer>;
  else l.kernel = backward ? norm_bwd_odd_kernel<T, 1024, 16, kLayer> : norm_fwd_odd_kernel<T, 1024, 16, kLayer>;
  l.threads = round32((dim + per - 1) / per);
  // as many blocks an SM as their registers allow: 1,024 threads of the forward kernel, 672 of the backward one, with 16 elements a
  // thread 512 (or 1,024 of either)
  const int by_registers = (per == 16 ? 512 : backward ? 672 : 1024) / l.threads;
  int per_sm = by_registers < 1 ? 1 : by_registers;
  const int stage = (backward ? 2 : 1) * odd_row_bytes(dim * static_cast<int>(sizeof(T)));
  l.stages = 3;
  while (l.stages > 1 && per_sm * (l.stages * stage + 2048) > kMostShared) --l.stages;
  l.shared = l.stages * stage;
  const int64_t most = static_cast<int64_t>(kSms) * per_sm;
  l.blocks = rows < most ? rows : most;
  return l;
}

// Vectors of a lane, warps of a row and rows of a team in the forward pass: 64 registers hold what is under way, 16 vectors of bf16 or 8
// of fp32. Few rows go one to a team, so that they are spread over the SMs.
template <typename T, bool kLayer>
Launch fwd_launch(int dim, int64_t rows) {
  const int n = dim / 8;
  Launch l;
  int per_block = 0;
  auto use = [&](auto lanes, auto vecs, auto warps, auto together) {
    constexpr int L = decltype(lanes)::value, V = decltype(vecs)::value, W = decltype(warps)::value, R = decltype(together)::value;
    const int teams = fwd_threads(W) / (L * W);
    const bool spread = R > 1 && rows < static_cast<int64_t>(kSms) * 4 * teams * R;
    if constexpr (W > 1) l.kernel = spread ? norm_fwd_kernel<T, L, V, W, 1, kLayer> : norm_fwd_kernel<T, L, V, W, R, kLayer>;
    else l.kernel = norm_fwd_kernel<T, L, V, W, R, kLayer>;
    l.threads = fwd_threads(W), per_block = teams * (W > 1 && spread ? 1 : R);
  };
#define NSP_USE(L, V, W, R) use(std::integral_constant<int, L>{}, std::integral_constant<int, V>{}, std::integral_constant<int, W>{}, std::integral_constant<int, R>{})
  if (n <= 8) NSP_USE(8, 1, 1, 4);
  else if (n <= 16) NSP_USE(8, 2, 1, 2);
  else if (n <= 32) NSP_USE(16, 2, 1, 2);
  else if (n <= 64) NSP_USE(32, 2, 1, 2);
  else if (n <= 128) NSP_USE(32, 4, 1, 2);
  else if (n <= 256) NSP_USE(32, 4, 2, 2);
  else if (n <= 512) NSP_USE(32, 4, 4, 2);
  else if (n <= 1024) {  // one barrier for four warps (bf16, 16,384 rows: 105 us; eight warps of four vectors 116)
    if constexpr (sizeof(T) == 2) NSP_USE(32, 8, 4, 2);
    else NSP_USE(32, 4, 8, 2);
  }
  else if (sizeof(T) == 4 || rows <= 2 * kSms) NSP_USE(32, 4, 16, 1);  // fp32, and few rows (one row of 16,384 bf16: 3.7 us, with half the warps 4.6)
  else if constexpr (sizeof(T) == 2) NSP_USE(32, 8, 8, 1);
#undef NSP_USE
  l.blocks = (rows + per_block - 1) / per_block;
  return l;
}

template <typename T, int kKind>
Launch bwd_launch(int dim, int64_t rows) {
  const int n = dim / 8;
  Launch l;
  int64_t most = 0;
  int rows_of_block = 0;
  auto brief = [&](void (*k)(const NormArgs), int lanes, int rows_of_team) {
    l.kernel = k, l.threads = 256, rows_of_block = 256 / lanes * rows_of_team, most = 2 * kSms;
  };
  if (n <= 8) brief(norm_bwd_short_kernel<T, 8, 1, 4, kKind>, 8, 4);
  else if (n <= 16) brief(norm_bwd_short_kernel<T, 8, 2, 2, kKind>, 8, 2);
  else if (n <= 32) brief(norm_bwd_short_kernel<T, 16, 2, 2, kKind>, 16, 2);
  else if (n <= 64) brief(norm_bwd_short_kernel<T, 32, 2, 2, kKind>, 32, 2);
  else {
    const int vecs = n > 1536 ? 4 : n > 1024 ? 3 : 2;
    if (n > 1536) l.kernel = norm_bwd_long_kernel<T, 512, 4, kKind>;
    else if (n > 1024) l.kernel = norm_bwd_long_kernel<T, 512, 3, kKind>;
    else if (n > 512) l.kernel = norm_bwd_long_kernel<T, 512, 2, kKind>;
    else l.kernel = norm_bwd_long_kernel<T, 256, 2, kKind>;
    l.threads = n > 512 ? 512 : 256;
    l.team = vecs == 3 ? l.threads : round32((n + vecs - 1) / vecs);
    rows_of_block = l.threads / l.team;
    const int stage = 2 * l.threads * vecs * 8 * static_cast<int>(sizeof(T));
    // two blocks an SM where three stages of each fit
    int per_sm = l.threads > 256 ? 1 : 2;
    while (per_sm > 1 && per_sm * (3 * stage + 2048) > kMostShared) --per_sm;
    l.stages = 3;
    while (l.stages > 1 && l.stages * stage + 2048 > kMostShared) --l.stages;
    l.shared = l.stages * stage;
    most = static_cast<int64_t>(per_sm) * kSms;
  }
  const int64_t need = (rows + rows_of_block - 1) / rows_of_block;
  l.blocks = need < most ? need : most;
  return l;
}

Launch launch_of(bool vectors, int dim, int64_t rows, int dtype, bool layer, bool bias, bool backward) {
  const bool f32 = dtype == NSP_F32;
  if (!vectors) {
    if (f32) return layer ? element_launch<float, true>(dim, rows, backward) : element_launch<float, false>(dim, rows, backward);
    return layer ? element_launch<__nv_bfloat16, true>(dim, rows, backward) : element_launch<__nv_bfloat16, false>(dim, rows, backward);
  }
  if (!backward) {
    if (f32) return layer ? fwd_launch<float, true>(dim, rows) : fwd_launch<float, false>(dim, rows);
    return layer ? fwd_launch<__nv_bfloat16, true>(dim, rows) : fwd_launch<__nv_bfloat16, false>(dim, rows);
  }
  if (f32) return layer ? bwd_launch<float, kLayerBias>(dim, rows) : bias ? bwd_launch<float, kRmsBias>(dim, rows) : bwd_launch<float, kRms>(dim, rows);
  return layer ? bwd_launch<__nv_bfloat16, kLayerBias>(dim, rows)
               : bias ? bwd_launch<__nv_bfloat16, kRmsBias>(dim, rows) : bwd_launch<__nv_bfloat16, kRms>(dim, rows);
}

cudaError_t launch(const Launch& l, NormArgs& a, cudaStream_t st) {
  if (l.shared > 40 * 1024) {  // with what the kernel has of its own, more than the 48 KB of an ordinary launch
    // The same value in every call, whatever this one needs: the attribute is the kernel's, and a smaller one would make the launch of
    // another thread fail that has just set what it needs.
    const cudaError_t e = cudaFuncSetAttribute(l.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared - kStaticShared);
    if (e != cudaSuccess) return cudaGetLastError(), e;
  }
  a.stages = l.stages, a.team = l.team;
  nsp::count_launches(1);
  return nsp::launch_chained_if(true, l.kernel, static_cast<unsigned>(l.blocks), l.threads, l.shared, st, a);
}

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
  return launch(launch_of(vectors, dim, a.rows, dtype, kind == NSP_NORM_LAYER, false, false), a, static_cast<cudaStream_t>(stream)) ==
                 cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
}

extern "C" int nsp_norm_bwd_ws_bytes(int64_t rows, int32_t dim, size_t* bytes) {
  if (!bytes || rows < 0 || dim < 1) return NSP_ERR_INVALID_ARG;
  if (dim > NSP_NORM_MAX_DIM || rows > INT32_MAX) return NSP_ERR_UNSUPPORTED;
  int64_t most = 0;  // of any kernel for rows of that length
  for (int dtype : {NSP_BF16, NSP_F32}) {
    for (bool vectors : {false, true}) {
      if (vectors && dim % 8) continue;
      const int64_t n = launch_of(vectors, dim, rows, dtype, true, true, true).blocks;
      most = n > most ? n : most;
    }
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
    const Launch l = launch_of(vectors, dim, a.rows, dtype, layer, dbias != nullptr, true);
    blocks = static_cast<int>(l.blocks);
    if (grads && (!ws || !aligned(ws, 16) || ws_bytes < 2 * sizeof(float) * static_cast<size_t>(blocks) * dim)) return NSP_ERR_WORKSPACE;
    a.w = weight, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.part = static_cast<float*>(ws);
    a.inner = inner, a.dim = dim, a.w_f32 = w_dtype == NSP_F32, a.want_grads = grads, a.inv_dim = 1.f / static_cast<float>(dim);
    if (launch(l, a, st) != cudaSuccess) return NSP_ERR_CUDA;
  }
  if (!grads) return NSP_OK;
  nsp::count_launches(1);
  const int warps = blocks >= 256 ? 32 : blocks >= 16 ? 16 : blocks > 1 ? blocks : 1;
  return nsp::launch_chained_if(true, norm_grads_kernel, 2 * ((dim + 31) / 32), 32 * warps, 0, st, static_cast<const float*>(ws), blocks, dim,
                                dweight, dbias) == cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
}
