// Rotary positions of queries and keys, and the way back of their gradients: the step between the projections and the
// attention of a node (paper Sec. 4.1.2, non-attention work of a layer). A pair (a, b) of a head at position p becomes
//     (a c - b s, b c + a s),   c = m cos(p f), s = m sin(p f),
// f the pair's frequency and m a factor on both; the gradient of that is the same rotation with -s. HBM-bound: every element is
// read once and written once, 6 flop per pair.
//
// The angle. p f reaches 10^5 radians and more, where 32 bits leave two or three digits of the angle. A frequency is therefore
// kept as a fraction of a turn in 64-bit fixed point, F = round(2^64 frac(f / 2 pi)): p F modulo 2^64 is the exact fractional
// turn of p F (an integer product drops whole turns by itself), its upper 32 bits as a signed number are the angle within half a
// turn, 2^-32 of a turn apart, and sincospif takes it from there. The error is p * 2^-65 of a turn, for any p a batch can
// have below the rounding of the cosine.
//
// Work. A thread owns V pairs of a head (one 16-byte load for each half of them in bf16) of up to 16 neighbouring heads of one
// token: the sines and cosines are computed once for these, and up to four heads' loads are under way at a time. Groups of J
// threads, one per slot of a head, cover all slots of a (token, heads) piece.
#include <cmath>
#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "nsp_internal.cuh"
#include "sm100_ptx.cuh"

using nsp::grid_launch_dependents;
using nsp::grid_wait_predecessor;
using nsp::pack_bf16x2;

namespace {

constexpr int kMaxPairs = NSP_ROPE_MAX_ROT / 2;
constexpr int kMostHeads = 16;  // heads of a thread

struct RopeTensor {
  const void* x;
  void* y;
  const int64_t* pos;
  int64_t x_tok, x_head, y_tok, y_head;  // elements
  int64_t block0;                        // first block of the tensor
  uint32_t tokens;
  int32_t heads, per, chunks;  // `per` heads of a thread, `chunks` such pieces of a token
  int32_t f32;
};

struct RopeArgs {
  uint64_t freq[kMaxPairs];  // turns per position, 64-bit fixed point
  RopeTensor t[NSP_ROPE_MAX_TENSORS];
  int32_t n, pairs;
  int32_t slots, rot_slots, per_block;  // threads of a group, those that rotate, groups of a block
  int32_t dim, rot;
  float magnitude, sin_sign;
};

// V elements as they are in memory
template <typename T, int V>
struct Raw {
  static constexpr int kBytes = V * static_cast<int>(sizeof(T));
  static constexpr int kWords = kBytes / 4;
  uint32_t w[kWords ? kWords : 1];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 q = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + 16 * i);
        w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      w[0] = q.x, w[1] = q.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i)
        *reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) + 16 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else if constexpr (kBytes == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else if constexpr (kBytes == 4) {
      *reinterpret_cast<uint32_t*>(p) = w[0];
    } else {
      *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[V]) {  // the one rounding of an output, to nearest
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = __float_as_uint(v[i]);
    } else if constexpr (V == 1) {
      w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    }
  }
};

template <typename T, int V, bool kHalf>
__device__ __forceinline__ void rope_piece(const RopeTensor& t, const uint64_t* freq, uint32_t token, int h0, int slot, int rot_slots,
                                           int dim, int rot, float magnitude, float sin_sign) {
  constexpr int kBatch = V * sizeof(T) > 16 ? 2 : 4;  // heads whose loads are under way together
  const int n = min(t.per, t.heads - h0);
  const T* x = static_cast<const T*>(t.x) + static_cast<int64_t>(token) * t.x_tok + h0 * t.x_head;
  T* y = static_cast<T*>(t.y) + static_cast<int64_t>(token) * t.y_tok + h0 * t.y_head;
  // the two vectors of a slot: V first and V second elements of pairs, or V pairs of neighbours; two vectors of the rest
  const bool rotates = slot < rot_slots;
  int a_at, b_at;
  bool second = true;
  if (rotates) {
    a_at = kHalf ? slot * V : 2 * slot * V;
    b_at = kHalf ? rot / 2 + slot * V : (2 * slot + 1) * V;
  } else {
    a_at = rot + 2 * (slot - rot_slots) * V;
    b_at = a_at + V;
    second = b_at < dim;
  }
  const uint64_t p = t.pos ? static_cast<uint64_t>(t.pos[token]) : token;
  float c[V], s[V];
  for (int first = 0; first < n; first += kBatch, x += kBatch * t.x_head, y += kBatch * t.y_head) {
    Raw<T, V> a[kBatch], b[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (first + i < n) {
        a[i].load(x + i * t.x_head + a_at);
        if (second) b[i].load(x + i * t.x_head + b_at);
      }
    }
    if (rotates) {
      if (first == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int32_t turn = static_cast<int32_t>((p * freq[slot * V + i]) >> 32);
          sincospif(static_cast<float>(turn) * 0x1p-31f, &s[i], &c[i]);
          c[i] *= magnitude;
          s[i] *= sin_sign;
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        float u[V], v[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          // pair k of the slot; neighbours: elements 2 k and 2 k + 1 of the two vectors
          const int e = 2 * k;
          const float p0 = kHalf ? a[i].get(k) : (e < V ? a[i].get(e % V) : b[i].get(e % V));
          const float p1 = kHalf ? b[i].get(k) : (e + 1 < V ? a[i].get((e + 1) % V) : b[i].get((e + 1) % V));
          const float q0 = p0 * c[k] - p1 * s[k], q1 = p1 * c[k] + p0 * s[k];
          if (kHalf) {
            u[k] = q0, v[k] = q1;
          } else {
            (e < V ? u : v)[e % V] = q0;
            (e + 1 < V ? u : v)[(e + 1) % V] = q1;
          }
        }
        a[i].set(u);
        b[i].set(v);
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (first + i < n) {
        a[i].store(y + i * t.y_head + a_at);
        if (second) b[i].store(y + i * t.y_head + b_at);
      }
    }
  }
}

// kF32: tensors of either type; otherwise all of them bf16
template <int V, bool kHalf, bool kF32>
__global__ void __launch_bounds__(V == 1 ? 512 : 256, V == 1 ? 1 : kF32 ? 2 : 3) rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ uint64_t freq[kMaxPairs];
  for (int i = threadIdx.x; i < a.pairs; i += blockDim.x) freq[i] = a.freq[i];
  grid_wait_predecessor();
  grid_launch_dependents();
  __syncthreads();
  int k = 0;
  while (k + 1 < a.n && static_cast<int64_t>(blockIdx.x) >= a.t[k + 1].block0) ++k;
  const RopeTensor& t = a.t[k];
  const int slot = static_cast<int>(threadIdx.x) % a.slots, g = static_cast<int>(threadIdx.x) / a.slots;
  const int64_t group = (blockIdx.x - t.block0) * a.per_block + g;
  if (group >= static_cast<int64_t>(t.tokens) * t.chunks) return;
  const uint32_t token = static_cast<uint32_t>(group) / static_cast<uint32_t>(t.chunks);  // groups of a tensor: below 2^32
  const int h0 = static_cast<int>(static_cast<uint32_t>(group) - token * t.chunks) * t.per;
  if (kF32 && t.f32)
    rope_piece<float, V, kHalf>(t, freq, token, h0, slot, a.rot_slots, a.dim, a.rot, a.magnitude, a.sin_sign);
  else
    rope_piece<__nv_bfloat16, V, kHalf>(t, freq, token, h0, slot, a.rot_slots, a.dim, a.rot, a.magnitude, a.sin_sign);
}

// Rows [tokens, heads] of `dim` elements at these strides do not overlap.
bool distinct(int64_t tokens, int64_t heads, int64_t dim, int64_t s_tok, int64_t s_head) {
  if (tokens <= 1) return heads <= 1 || s_head >= dim;
  if (heads <= 1) return s_tok >= dim;
  return s_tok >= s_head ? s_head >= dim && s_tok >= (heads - 1) * s_head + dim : s_tok >= dim && s_head >= (tokens - 1) * s_tok + dim;
}
constexpr int64_t kMostStride = int64_t{1} << 31;  // elements: with 2^31 rows at most, offsets stay inside 64 bits

}  // namespace

extern "C" int nsp_rope_frequencies(int32_t rot_dim, double base, const nsp_rope_scaling_t* scaling, double* inv_freq, float* magnitude) {
  if (!inv_freq || !magnitude || rot_dim < 2 || rot_dim % 2 || rot_dim > NSP_ROPE_MAX_ROT || !(base > 1.0) || !std::isfinite(base))
    return NSP_ERR_INVALID_ARG;
  const int n = rot_dim / 2;
  const int kind = scaling ? scaling->kind : NSP_ROPE_PLAIN;
  if (kind < NSP_ROPE_PLAIN || kind > NSP_ROPE_PARTS) return NSP_ERR_INVALID_ARG;
  double scale = 1.0;
  if (kind != NSP_ROPE_PLAIN) {
    scale = scaling->scale;
    if (!(scale >= 1.0) || !std::isfinite(scale)) return NSP_ERR_INVALID_ARG;
  }
  if (kind == NSP_ROPE_BASE && rot_dim > 2) base *= std::pow(scale, rot_dim / (rot_dim - 2.0));
  double lo = 0, hi = 0;
  if (kind == NSP_ROPE_PARTS) {
    if (!(scaling->fast_turns > scaling->slow_turns) || !(scaling->slow_turns > 0) || !std::isfinite(scaling->fast_turns) ||
        !(scaling->trained_tokens > 0) || !std::isfinite(scaling->trained_tokens))
      return NSP_ERR_INVALID_ARG;
    auto pair_of = [&](double turns) {
      return rot_dim * std::log(scaling->trained_tokens / (turns * 2 * M_PI)) / (2 * std::log(base));
    };
    lo = std::fmax(std::floor(pair_of(scaling->fast_turns)), 0.0);
    hi = std::fmin(std::ceil(pair_of(scaling->slow_turns)), rot_dim - 1.0);
  }
  for (int i = 0; i < n; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    if (kind == NSP_ROPE_LINEAR) {
      inv_freq[i] = f / scale;
    } else if (kind == NSP_ROPE_PARTS) {
      const double pressed = std::fmin(std::fmax((i - lo) / std::fmax(hi - lo, 1e-3), 0.0), 1.0);
      inv_freq[i] = f / scale * pressed + f * (1 - pressed);
    } else {
      inv_freq[i] = f;
    }
  }
  *magnitude = kind == NSP_ROPE_PARTS && scale > 1 ? static_cast<float>(0.1 * std::log(scale) + 1.0) : 1.0f;
  return NSP_OK;
}

extern "C" int nsp_rope(const nsp_rope_tensor_t* tensors, int32_t n_tensors, int32_t head_dim, int32_t rot_dim, int32_t layout,
                        const double* inv_freq, float magnitude, int32_t inverse, void* stream) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !inv_freq || head_dim < 1 || rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim ||
      (layout != NSP_ROPE_HALF && layout != NSP_ROPE_INTERLEAVED) || !std::isfinite(magnitude))
    return NSP_ERR_INVALID_ARG;
  if (n_tensors > NSP_ROPE_MAX_TENSORS || rot_dim > NSP_ROPE_MAX_ROT || head_dim > NSP_ROPE_MAX_HEAD_DIM) return NSP_ERR_UNSUPPORTED;
  RopeArgs a;
  a.pairs = rot_dim / 2;
  for (int i = 0; i < a.pairs; ++i) {
    if (!std::isfinite(inv_freq[i])) return NSP_ERR_INVALID_ARG;
    // the 64 bits of mantissa of an x87 long double are those of the fixed point
    const long double turns = static_cast<long double>(inv_freq[i]) / 6.283185307179586476925286766559L;
    const long double fixed = std::roundl(std::ldexp(turns - std::floor(turns), 64));
    a.freq[i] = fixed >= 18446744073709551616.0L ? 0 : static_cast<uint64_t>(fixed);
  }
  int vec = 8;  // elements of a vector, as far as every tensor's addresses allow
  auto fits = [&](int v) { return a.pairs % v == 0 && rot_dim % v == 0 && head_dim % v == 0; };
  while (vec > 1 && !fits(vec)) vec = vec == 8 ? 4 : 1;
  bool copies = false, any_f32 = false;
  int64_t pieces = 0;  // (token, head)
  a.n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const nsp_rope_tensor_t& s = tensors[i];
    if (s.tokens < 0 || s.heads < 1 || (s.dtype != NSP_BF16 && s.dtype != NSP_F32)) return NSP_ERR_INVALID_ARG;
    for (int64_t stride : {s.x_token_stride, s.x_head_stride, s.y_token_stride, s.y_head_stride})
      if (stride < 0 || stride > kMostStride) return NSP_ERR_INVALID_ARG;
    if (s.tokens == 0) continue;
    if (s.tokens > INT32_MAX || s.heads > 65536 || s.tokens * s.heads > INT32_MAX) return NSP_ERR_UNSUPPORTED;
    const int size = s.dtype == NSP_F32 ? 4 : 2;
    if (!s.x || !s.y || reinterpret_cast<uintptr_t>(s.x) % size || reinterpret_cast<uintptr_t>(s.y) % size ||
        reinterpret_cast<uintptr_t>(s.positions) % 8)
      return NSP_ERR_INVALID_ARG;
    if (!distinct(s.tokens, s.heads, head_dim, s.y_token_stride, s.y_head_stride)) return NSP_ERR_INVALID_ARG;
    if (s.x == s.y && ((s.tokens > 1 && s.x_token_stride != s.y_token_stride) || (s.heads > 1 && s.x_head_stride != s.y_head_stride)))
      return NSP_ERR_INVALID_ARG;
    if (s.x != s.y) copies = true;
    if (s.dtype == NSP_F32) any_f32 = true;
    auto ok = [&](int v) {
      const uintptr_t bytes = static_cast<uintptr_t>(v * size > 16 ? 16 : v * size);
      auto stride = [&](int64_t e, int64_t count) { return count <= 1 || (e * size) % static_cast<int64_t>(bytes) == 0; };
      return reinterpret_cast<uintptr_t>(s.x) % bytes == 0 && reinterpret_cast<uintptr_t>(s.y) % bytes == 0 &&
             stride(s.x_token_stride, s.tokens) && stride(s.y_token_stride, s.tokens) && stride(s.x_head_stride, s.heads) &&
             stride(s.y_head_stride, s.heads);
    };
    while (vec > 1 && !(fits(vec) && ok(vec))) vec = vec == 8 ? 4 : 1;
    RopeTensor& t = a.t[a.n++];
    t.x = s.x, t.y = s.y, t.pos = s.positions;
    t.x_tok = s.x_token_stride, t.x_head = s.x_head_stride, t.y_tok = s.y_token_stride, t.y_head = s.y_head_stride;
    t.tokens = static_cast<uint32_t>(s.tokens), t.heads = s.heads, t.f32 = s.dtype == NSP_F32;
    pieces += s.tokens * s.heads;
  }
  if (a.n == 0) return NSP_OK;
  a.dim = head_dim, a.rot = rot_dim;
  a.rot_slots = a.pairs / vec;
  a.slots = a.rot_slots + (copies ? (head_dim - rot_dim + 2 * vec - 1) / (2 * vec) : 0);
  const int threads = vec == 1 ? 512 : 256;
  a.per_block = threads / a.slots;
  a.magnitude = magnitude;
  a.sin_sign = inverse ? -magnitude : magnitude;
  // Heads of a thread: as many as leave every SM its threads
  int per = kMostHeads;
  while (per > 1 && pieces * a.slots / per < 148 * 1024) per /= 2;
  int64_t blocks = 0;
  for (int i = 0; i < a.n; ++i) {
    RopeTensor& t = a.t[i];
    t.per = per < t.heads ? per : t.heads;
    t.chunks = (t.heads + t.per - 1) / t.per;
    t.block0 = blocks;
    blocks += (static_cast<int64_t>(t.tokens) * t.chunks + a.per_block - 1) / a.per_block;
  }
  if (blocks > INT32_MAX) return NSP_ERR_UNSUPPORTED;
  const bool half = layout == NSP_ROPE_HALF;
  auto pick = [&](auto v) {
    constexpr int V = decltype(v)::value;
    return any_f32 ? (half ? rope_kernel<V, true, true> : rope_kernel<V, false, true>)
                   : (half ? rope_kernel<V, true, false> : rope_kernel<V, false, false>);
  };
  void (*kernel)(const RopeArgs) = vec == 8 ? pick(std::integral_constant<int, 8>{})
                                   : vec == 4 ? pick(std::integral_constant<int, 4>{}) : pick(std::integral_constant<int, 1>{});
  nsp::count_launches(1);
  return nsp::launch_chained_if(true, kernel, static_cast<unsigned>(blocks), a.slots * a.per_block, 0, static_cast<cudaStream_t>(stream),
                                a) == cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
}
