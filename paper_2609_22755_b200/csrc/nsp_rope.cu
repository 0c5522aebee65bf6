// Rotary positions of queries and keys, and the way back of their gradients: the step between the projections and the
// attention of a node (paper Sec. 4.1.2, non-attention work of a layer). A pair (a, b) of a head at position p becomes
//     (a c - b s, b c + a s),   c = m cos(p f), s = m sin(p f),
// f the pair's frequency and m a factor on both; the gradient of that is the same rotation with -s. HBM-bound: every element is
// read once and written once, 6 flop per pair.
//
// The angle. p f reaches 10^5 radians and more, where 32 bits leave two or three digits of the angle. A frequency is therefore
// kept as a fraction of a turn in 64-bit fixed point, F = 2^64 frac(f / 2 pi): p F modulo 2^64 is the exact fractional
// turn of p F (an integer product drops whole turns by itself). Its upper 32 bits give the quarter turn and, as a signed number,
// the rest within an eighth; the lower ones are cut off. The error is 2^-32 of a turn from that cut, and |p| times the frequency's own: F has
// that of the product f / 2 pi in 64 bits and of the cut behind it, together below 2^-63 of a turn for |f| <= 2 pi (frequencies of several
// turns a position lose as many more bits as their whole turns take). Both are below the rounding of the cosine for |p| <= 2^36.
//
// Work. A thread owns V pairs of a head (one 16-byte load for each half of them in bf16) of up to 16 neighbouring heads of one
// token, or of all heads of q and of k where they are no more (a chain's upper nodes: 4 and 1): the sines and cosines are computed
// once for these, and up to four heads' loads are under way at a time. Groups of J threads, one per slot of a head, cover all
// slots of a (token, heads) piece.
#include <algorithm>
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
  int32_t joined;  // 1: its threads go on with the next tensor's heads of the token; that one has no blocks of its own
};

// Kernel parameters for up to kTensors tensors and kPairs frequencies: a launch copies them, and the common call needs a twelfth.
template <int kTensors, int kPairs>
struct RopeArgs {
  uint64_t freq[kPairs];  // turns per position, 64-bit fixed point
  RopeTensor t[kTensors];
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

// m cos and m sin of a turn in 64-bit fixed point (sin_m: m or -m). The rest of the angle behind its quarter turn, f in [-pi/4, pi/4],
// goes through polynomials in f^2 fitted for the smallest relative error by reweighted least squares (sine 3.8e-9, cosine 1.2e-10);
// in fp32 both are within 1.7 * 2^-24 of those of f. A third of the instructions of a general sincospi, which has to find the quarter turn of a
// float.
__device__ __forceinline__ void sincos_turn(uint64_t turn, float m, float sin_m, float& c, float& s) {
  const uint32_t top = static_cast<uint32_t>(turn >> 32), quarter = (top + 0x20000000u) >> 30;
  const float f = static_cast<float>(static_cast<int32_t>(top - (quarter << 30))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float f2 = f * f;
  float p = fmaf(f2, -0.00019515282684585036f, 0.00833216075923622f);
  p = fmaf(p, f2, -0.16666654609533538f);
  const float sine = fmaf(p, f2 * f, f);
  float q = fmaf(f2, 2.4433155139662247e-05f, -0.0013887316236525606f);
  q = fmaf(q, f2, 0.041666645682576074f);
  q = fmaf(q, f2, -0.5f);
  const float cosine = fmaf(q, f2, 1.f);
  const bool odd = quarter & 1;
  const float u = odd ? sine : cosine, v = odd ? cosine : sine;
  // quarter 0: (cos, sin), 1: (-sin, cos), 2: (-cos, -sin), 3: (sin, -cos)
  c = __uint_as_float(__float_as_uint(u) ^ (((quarter + 1) & 2) << 30)) * m;
  s = __uint_as_float(__float_as_uint(v) ^ ((quarter & 2) << 30)) * sin_m;
}

// What a thread has of every head: the two vectors of its slot, V first and V second elements of pairs, or V pairs of neighbours; or
// two vectors of the rest, copied.
template <int V, bool kHalf>
struct Slot {
  int a_at, b_at;
  bool rotates, second;
  __device__ __forceinline__ Slot(int slot, int rot_slots, int dim, int rot) : rotates(slot < rot_slots), second(true) {
    if (rotates) {
      a_at = kHalf ? slot * V : 2 * slot * V;
      b_at = kHalf ? rot / 2 + slot * V : (2 * slot + 1) * V;
    } else {
      a_at = rot + 2 * (slot - rot_slots) * V;
      b_at = a_at + V;
      second = b_at < dim;
    }
  }
};

template <typename T, int V, bool kHalf, typename Angles>
__device__ __forceinline__ void rope_heads(const RopeTensor& t, uint32_t token, int h0, int n, const Slot<V, kHalf>& at, const float (&c)[V],
                                           const float (&s)[V], Angles angles) {
  constexpr int kBatch = V * sizeof(T) > 16 ? 2 : 4;  // heads whose loads are under way together
  const T* x = static_cast<const T*>(t.x) + static_cast<int64_t>(token) * t.x_tok + h0 * t.x_head;
  T* y = static_cast<T*>(t.y) + static_cast<int64_t>(token) * t.y_tok + h0 * t.y_head;
  for (int first = 0; first < n; first += kBatch, x += kBatch * t.x_head, y += kBatch * t.y_head) {
    Raw<T, V> a[kBatch], b[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (first + i < n) {
        a[i].load(x + i * t.x_head + at.a_at);
        if (at.second) b[i].load(x + i * t.x_head + at.b_at);
      }
    }
    if (at.rotates) {
      if (first == 0) angles();  // while the first loads are under way
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
        a[i].store(y + i * t.y_head + at.a_at);
        if (at.second) b[i].store(y + i * t.y_head + at.b_at);
      }
    }
  }
}

// kF32: tensors of either type; otherwise all of them bf16
template <int V, bool kHalf, bool kF32, typename Args>
__global__ void __launch_bounds__(V == 1 ? 512 : 256, V == 1 ? 1 : kF32 ? 2 : 3) rope_kernel(const __grid_constant__ Args a) {
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
  const Slot<V, kHalf> at(slot, a.rot_slots, a.dim, a.rot);
  const uint64_t p = t.pos ? static_cast<uint64_t>(t.pos[token]) : token;
  float c[V], s[V];
  auto angles = [&]() {
#pragma unroll
    for (int i = 0; i < V; ++i) sincos_turn(p * freq[slot * V + i], a.magnitude, a.sin_sign, c[i], s[i]);
  };
  auto heads = [&](const RopeTensor& t, int h0, auto first) {
    if (kF32 && t.f32)
      rope_heads<float, V, kHalf>(t, token, h0, min(t.per, t.heads - h0), at, c, s, first);
    else
      rope_heads<__nv_bfloat16, V, kHalf>(t, token, h0, min(t.per, t.heads - h0), at, c, s, first);
  };
  heads(t, h0, angles);
  if (t.joined) heads(a.t[k + 1], 0, [] {});
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
  RopeArgs<NSP_ROPE_MAX_TENSORS, kMaxPairs> a;
  a.pairs = rot_dim / 2;
  for (int i = 0; i < a.pairs; ++i) {
    if (!std::isfinite(inv_freq[i])) return NSP_ERR_INVALID_ARG;
    // the 64 bits of mantissa of an x87 long double are those of the fixed point
    long double turns = static_cast<long double>(inv_freq[i]) * 0.159154943091895335768883763372514362L;
    if (turns < 0 || turns >= 1) turns -= std::floor(turns);
    turns *= 18446744073709551616.0L;
    a.freq[i] = turns >= 18446744073709551615.0L ? 0 : static_cast<uint64_t>(turns);
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
    t.joined = 0;
    if (i > 0 && per == kMostHeads && !a.t[i - 1].joined && a.t[i - 1].pos == t.pos && a.t[i - 1].tokens == t.tokens &&
        (i < 2 || !a.t[i - 2].joined) && a.t[i - 1].heads + t.heads <= kMostHeads)
      a.t[i - 1].joined = 1;
    else
      blocks += (static_cast<int64_t>(t.tokens) * t.chunks + a.per_block - 1) / a.per_block;
  }
  if (blocks > INT32_MAX) return NSP_ERR_UNSUPPORTED;
  const bool half = layout == NSP_ROPE_HALF;
  const auto launch = [&](const auto& args) {
    using Args = std::decay_t<decltype(args)>;
    auto pick = [&](auto v) -> void (*)(const Args) {
      constexpr int V = decltype(v)::value;
      return any_f32 ? (half ? rope_kernel<V, true, true, Args> : rope_kernel<V, false, true, Args>)
                     : (half ? rope_kernel<V, true, false, Args> : rope_kernel<V, false, false, Args>);
    };
    void (*kernel)(const Args) = vec == 8 ? pick(std::integral_constant<int, 8>{})
                                 : vec == 4 ? pick(std::integral_constant<int, 4>{}) : pick(std::integral_constant<int, 1>{});
    nsp::count_launches(1);
    return nsp::launch_chained_if(true, kernel, static_cast<unsigned>(blocks), a.slots * a.per_block, 0, static_cast<cudaStream_t>(stream),
                                  args) == cudaSuccess ? NSP_OK : NSP_ERR_CUDA;
  };
  constexpr int kFew = 4, kFewPairs = 64;
  if (a.n > kFew || a.pairs > kFewPairs) return launch(a);
  RopeArgs<kFew, kFewPairs> few;
  std::copy_n(a.freq, a.pairs, few.freq);
  std::copy_n(a.t, a.n, few.t);
  few.n = a.n, few.pairs = a.pairs, few.slots = a.slots, few.rot_slots = a.rot_slots, few.per_block = a.per_block;
  few.dim = a.dim, few.rot = a.rot, few.magnitude = a.magnitude, few.sin_sign = a.sin_sign;
  return launch(few);
}
