// st_norm_rope: what stands between a layer's projections and the calls that
// take its queries and keys.  Each head of a row is normed by its root mean
// square, x / sqrt(mean x^2 + eps) w, and its first dimensions are rotated by the
// row's position, in one pass, in 32 bits, rounded once at the end.
//
// Angles.  Pair i turns by pos f_i; in turns of 2 pi, pos f_i / 2 pi, of which only
// the fraction counts.  f_i / 2 pi is given as a 64-bit fixed-point fraction, so
// the low 64 bits of its product with the position are the fraction itself, off
// by 2^-64 pos: far positions lose nothing (in 32 bits an angle of 131072 rad is
// off by 0.008).
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/st.h"
#include "kernels.cuh"

namespace st {

namespace {

struct RopeParams {
  const void* q;
  const void* k;
  const int32_t* positions;
  const uint64_t* turns;
  const void* q_weight;
  const void* k_weight;
  __nv_bfloat16* q_out;
  __nv_bfloat16* k_out;
  int64_t q_layer, q_row, k_layer, k_row;  // strides of the inputs, in elements
  int32_t n_rows, Hq, Hkv, rotary, interleaved;
  float eps;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// cos and sin of pair i at a position.
__device__ __forceinline__ float2 turn_of(uint64_t turns, int32_t pos) {
  const uint64_t t = turns * (uint64_t)(int64_t)pos;
  float s, c;
  sincospif((float)(int32_t)(t >> 32) * 0x1p-31f, &s, &c);
  return make_float2(c, s);
}

constexpr int kThreads = 256;
constexpr int kMaxRows = 4;  // of a block

// 8 values as they lie in global memory.
template <typename T>
struct Raw {
  uint4 x[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* from) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) x[i] = reinterpret_cast<const uint4*>(from)[i];
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(reinterpret_cast<const T*>(x)[i]);
  }
};

__device__ __forceinline__ void store8(__nv_bfloat16* y, const float* v) {
  uint4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 two = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    reinterpret_cast<uint32_t*>(&a)[i] = *reinterpret_cast<const uint32_t*>(&two);
  }
  *reinterpret_cast<uint4*>(y) = a;
}

// A block has `rows` rows (blockIdx.x), a part of their heads (blockIdx.z) and every
// gridDim.y-th layer from blockIdx.y on.  The rows' cosines and sines go to shared memory
// once for all of their heads and those layers.  A head has D / 16 threads, each
// with two pieces of 8 dimensions that are each other's partners (or neither is
// rotated), so that a value is read once, the norm is a few shuffles and the
// rotation is a thread's own.
template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const RopeParams p, int rows, int L) {
  constexpr int kPer = D / 16, kGroups = kThreads / kPer;
  __shared__ __align__(16) float2 turn[kMaxRows][D / 2];
  griddep_wait();
  griddep_launch_dependents();
  const int row0 = blockIdx.x * rows, n = min(rows, p.n_rows - row0), half = p.rotary / 2;
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int r = i / half, pair = i - r * half;
    turn[r][pair] = turn_of(p.turns[pair], p.positions[row0 + r]);
  }
  __syncthreads();
  const int c = threadIdx.x % kPer, pieces = p.rotary / 8;
  const uint32_t mates = ((1u << kPer) - 1) << (threadIdx.x % 32 / kPer * kPer);  // the threads of a head
  // this thread's pieces of a head
  int a = c, b = c + kPer;
  bool turned = 8 * a < p.rotary;
  if constexpr (!kInterleaved) {
    if (c < pieces / 2) b = c + pieces / 2;
    else a = pieces + 2 * (c - pieces / 2), b = a + 1, turned = false;
  }
  const int heads = p.Hq + p.Hkv, per = (heads + gridDim.z - 1) / gridDim.z;
  const int h0 = blockIdx.z * per, hn = min(per, heads - h0);
  for (int layer = blockIdx.y; layer < L; layer += gridDim.y) {
    auto place = [&](int task, int* r, int* row, int* head) -> bool {  // whether it is one of the queries
      *r = task / hn;
      *row = row0 + *r;
      const int h = h0 + task - *r * hn;
      *head = h < p.Hq ? h : h - p.Hq;
      return h < p.Hq;
    };
    Raw<T> raw[2];  // the next head's values, on their way while this one is turned
    auto fetch = [&](int task) {
      int r, row, head;
      const bool is_q = place(task, &r, &row, &head);
      const T* x = static_cast<const T*>(is_q ? p.q : p.k) + layer * (is_q ? p.q_layer : p.k_layer) +
                   row * (is_q ? p.q_row : p.k_row) + (int64_t)head * D;
      raw[0].load(x + 8 * a);
      raw[1].load(x + 8 * b);
    };
    if ((int)threadIdx.x / kPer < n * hn) fetch(threadIdx.x / kPer);
    for (int task = threadIdx.x / kPer; task < n * hn; task += kGroups) {
      float v[16];
      raw[0].values(v);
      raw[1].values(v + 8);
      if (task + kGroups < n * hn) fetch(task + kGroups);
      int r, row, head;
      const bool is_q = place(task, &r, &row, &head);
      const T* w = static_cast<const T*>(is_q ? p.q_weight : p.k_weight);
      if (w) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += v[i] * v[i];
#pragma unroll
        for (int o = 1; o < kPer; o *= 2) sum += __shfl_xor_sync(mates, sum, o);
        const float f = rsqrtf(sum / D + p.eps);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          Raw<T> weights;
          weights.load(w + layer * D + 8 * (e ? b : a));
          float wv[8];
          weights.values(wv);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[8 * e + i] *= f * wv[i];
        }
      }
      if constexpr (kInterleaved) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int first = 4 * (e ? b : a);  // pair of the piece
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (first + i >= half) break;
            const float2 t = turn[r][first + i];
            const float y = v[8 * e + 2 * i], z = v[8 * e + 2 * i + 1];
            v[8 * e + 2 * i] = y * t.x - z * t.y;
            v[8 * e + 2 * i + 1] = z * t.x + y * t.y;
          }
        }
      } else if (turned) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float4 t = *reinterpret_cast<const float4*>(&turn[r][8 * a + i]);
          const float y0 = v[i], z0 = v[8 + i], y1 = v[i + 1], z1 = v[9 + i];
          v[i] = y0 * t.x - z0 * t.y, v[8 + i] = z0 * t.x + y0 * t.y;
          v[i + 1] = y1 * t.z - z1 * t.w, v[9 + i] = z1 * t.z + y1 * t.w;
        }
      }
      __nv_bfloat16* out = (is_q ? p.q_out : p.k_out) +
                           (((int64_t)layer * p.n_rows + row) * (is_q ? p.Hq : p.Hkv) + head) * D;
      store8(out + 8 * a, v);
      store8(out + 8 * b, v + 8);
    }
  }
}

// A rotated part that is no multiple of 16 dimensions, in halves: a pair's two values
// are not in pieces of 8, so a warp has a head and its normed values meet in
// shared memory.  Loads of 2 bytes and a block a row bound it: 8191 rows of 64/8 heads of 128, four
// layers, 443 us where a multiple of 16 takes 215.  Kept simple, since such parts are rare.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) norm_rope_odd_kernel(const RopeParams p) {
  __shared__ float normed[kThreads / 32][D];
  __shared__ float2 turn[D / 2];
  griddep_wait();
  griddep_launch_dependents();
  const int row = blockIdx.x, layer = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int half = p.rotary / 2;
  for (int i = threadIdx.x; i < half; i += kThreads) turn[i] = turn_of(p.turns[i], p.positions[row]);
  __syncthreads();
  for (int h = warp; h < p.Hq + p.Hkv; h += kThreads / 32) {
    const bool is_q = h < p.Hq;
    const int head = is_q ? h : h - p.Hq;
    const T* x = static_cast<const T*>(is_q ? p.q : p.k) + layer * (is_q ? p.q_layer : p.k_layer) +
                 row * (is_q ? p.q_row : p.k_row) + (int64_t)head * D;
    const T* w = static_cast<const T*>(is_q ? p.q_weight : p.k_weight);
    float v[D / 32], sum = 0.f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      v[e] = to_float(x[e * 32 + lane]);
      sum += v[e] * v[e];
    }
    if (w) {
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float f = rsqrtf(sum / D + p.eps);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) v[e] *= f * to_float(w[layer * D + e * 32 + lane]);
    }
#pragma unroll
    for (int e = 0; e < D / 32; ++e) normed[warp][e * 32 + lane] = v[e];
    __syncwarp();
    __nv_bfloat16* out = (is_q ? p.q_out : p.k_out) +
                         (((int64_t)layer * p.n_rows + row) * (is_q ? p.Hq : p.Hkv) + head) * D;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      const int d = e * 32 + lane;
      float y = v[e];
      if (d < p.rotary) {
        const bool second = d >= half;
        const float2 t = turn[second ? d - half : d];
        const float other = normed[warp][second ? d - half : d + half];
        y = second ? y * t.x + other * t.y : y * t.x - other * t.y;
      }
      out[d] = __float2bfloat16_rn(y);
    }
    __syncwarp();
  }
}

template <typename T, int D>
cudaError_t launch_t(const RopeParams& p, int L, cudaStream_t s) {
  if (!p.interleaved && p.rotary % 16)
    return launch_chained(norm_rope_odd_kernel<T, D>, dim3(p.n_rows, L), dim3(kThreads), 0, s, p);
  // Many rows: four to a block, which goes through the layers with their sines.  Few:
  // a block for a row, a layer and as many heads as it has threads for, so that
  // nothing is done one after another.  32/8 heads of 128, us as few and as many (events, L2
  // flushed): 152 rows 8.8 and 10.9, 608 10.8 and 10.9, 1216 17.0 and 12.9, 2432 25.2 and 17.0;
  // 5 rows of 32 layers 8.8 and 10.9, 64 rows 23.2 and 17.0.
  const bool many = (int64_t)p.n_rows * L >= 4 * 152;
  const int rows = many ? kMaxRows : 1, blocks = (p.n_rows + rows - 1) / rows;
  constexpr int kGroups = kThreads / (D / 16);
  const int parts = many ? 1 : (p.Hq + p.Hkv + kGroups - 1) / kGroups;
  const int layers = many ? std::max(1, std::min(L, 152 * 8 / blocks)) : L;
  const dim3 grid(blocks, layers, parts);
  return p.interleaved ? launch_chained(norm_rope_kernel<T, D, true>, grid, dim3(kThreads), 0, s, p, rows, L)
                       : launch_chained(norm_rope_kernel<T, D, false>, grid, dim3(kThreads), 0, s, p, rows, L);
}

}  // namespace

}  // namespace st

extern "C" ST_API st_status st_norm_rope(const st_rope_config* c, const void* q, const void* k,
                                         const int32_t* positions, const uint64_t* turns, const void* q_weight,
                                         const void* k_weight, void* q_out, void* k_out, void* stream) {
  if (!c || c->n_layers < 1 || c->n_layers > 65535 || c->n_rows < 0 || c->n_q_heads < 0 || c->n_kv_heads < 0 ||
      c->n_q_heads > 65535 || c->n_kv_heads > 65535 || (c->head_dim != 64 && c->head_dim != 128) ||
      c->rotary_dim < 2 || c->rotary_dim > c->head_dim || c->rotary_dim % 2 || c->type < ST_BF16 || c->type > ST_F32 ||
      !(c->eps >= 0.f) || c->eps > 3e38f || (c->flags & ~ST_ROPE_INTERLEAVED))
    return ST_ERR_INVALID;
  if (c->n_rows == 0 || c->n_q_heads + c->n_kv_heads == 0) return ST_OK;
  const int size = c->type == ST_F32 ? 4 : 2;
  auto fits = [&](const void* in, const void* w, const void* out, int64_t layer, int64_t row, int heads) {
    if (heads == 0) return true;
    auto misaligned = [](const void* a) { return (uintptr_t)a % 16 != 0; };
    return in && out && !misaligned(in) && !misaligned(out) && !misaligned(w) && row >= 0 && layer >= 0 &&
           row * size % 16 == 0 && layer * size % 16 == 0;
  };
  if (!positions || !turns || (uintptr_t)positions % 4 || (uintptr_t)turns % 8 ||
      !fits(q, q_weight, q_out, c->q_layer_stride, c->q_row_stride, c->n_q_heads) ||
      !fits(k, k_weight, k_out, c->k_layer_stride, c->k_row_stride, c->n_kv_heads))
    return ST_ERR_INVALID;
  st::RopeParams p{};
  p.q = q;
  p.k = k;
  p.positions = positions;
  p.turns = turns;
  p.q_weight = q_weight;
  p.k_weight = k_weight;
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_out = static_cast<__nv_bfloat16*>(k_out);
  p.q_layer = c->q_layer_stride;
  p.q_row = c->q_row_stride;
  p.k_layer = c->k_layer_stride;
  p.k_row = c->k_row_stride;
  p.n_rows = c->n_rows;
  p.Hq = c->n_q_heads;
  p.Hkv = c->n_kv_heads;
  p.rotary = c->rotary_dim;
  p.interleaved = c->flags & ST_ROPE_INTERLEAVED;
  p.eps = c->eps;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto launch = [&](auto type) {
    using T = decltype(type);
    return c->head_dim == 128 ? st::launch_t<T, 128>(p, c->n_layers, s) : st::launch_t<T, 64>(p, c->n_layers, s);
  };
  const cudaError_t e = c->type == ST_BF16  ? launch(__nv_bfloat16())
                        : c->type == ST_F16 ? launch(__half())
                                            : launch(float());
  return e == cudaSuccess ? ST_OK : ST_ERR_CUDA;
}
