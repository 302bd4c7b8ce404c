// Rows into a pool that holds K and V in 4 bits, and out of it (format: kv4.cuh).
//
// A block has a page of one layer that the call touches, of one KV head after another:
// 2 D threads, one for each 8 values of a row.  K goes out as it is packed; V is
// packed along tokens, so its codes pass through shared memory.  The next head's
// rows are on their way while a head's are packed; with few pages each head has a
// block of its own.
//
// What bounds it: the instructions of a value (some 15: maximum, scaling, packing by
// token), with memory at two thirds.  12290 rows of 8 heads of 128 in four layers, into
// pages and back out: 59 and 45 us for 255 MB each way (4.3 and 5.7 TB/s; with a division a value
// and a block a head 119 and 66; with each value clamped, and tested for being a number, 75).
#include "kv4.cuh"

namespace st {

namespace {

// A page of the call: which branch, which of its rows, and the block it is in.
struct PageOfCall {
  int first, last;   // tokens [first, last) of the page are the call's
  int64_t row;       // the call's row of the page's token 0 (it may lie before the branch's first)
  int32_t block;
  int branch;
};

__device__ __forceinline__ PageOfCall page_of_call(const Kv4StoreParams& p, const Kv4Branch* brs, int page,
                                                   const int32_t* pages = nullptr) {
  int lo = 0, hi = p.n_br - 1;  // the last branch that begins at or before it
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (brs[mid].page0 <= page) lo = mid;
    else hi = mid - 1;
  }
  const Kv4Branch b = brs[lo];
  const int logical = b.start / kPageTokens + (page - b.page0);
  const int at = logical * kPageTokens - b.start;  // the branch's row at token 0
  PageOfCall r;
  r.first = max(0, -at);
  r.last = min(kPageTokens, b.n - at);
  r.row = (int64_t)b.row0 + at;
  r.block = pages ? pages[page] : p.table[(int64_t)b.slot * p.max_pages + logical];
  r.branch = lo;
  return r;
}

__device__ __forceinline__ float max_abs8(const uint4& x) {  // NaN aside
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  __nv_bfloat162 m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = w[i] & 0x7fff7fffu;
    m[i] = *reinterpret_cast<const __nv_bfloat162*>(&a);
  }
  const __nv_bfloat162 y = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
  return fmaxf(fmaxf(__low2float(y), __high2float(y)), 0.f);
}

// The same as bf16 bits, where an infinity is above all numbers and a NaN above it.
__device__ __forceinline__ uint32_t max_bits8(const uint4& x) {
  constexpr uint32_t kMagnitude = 0x7fff7fffu;
  const uint32_t m = __vmaxu2(__vmaxu2(x.x & kMagnitude, x.y & kMagnitude), __vmaxu2(x.z & kMagnitude, x.w & kMagnitude));
  return max(m & 0xffffu, m >> 16);
}
// Groups whose scale is rounded in steps of its own (the largest below 7 2^-14), at most 3840
// (above 7 3840), or that have what is no number; in the others |x / s| is below 7.5.
__device__ __forceinline__ bool unusual(uint32_t top) { return (top < 0x39e0u && top != 0) || top > 0x46d2u; }

// The codes of 8 values under a scale's inverse; `careful` where some group of the warp is unusual.
__device__ __forceinline__ void codes8(const uint4& x, float r, bool careful, uint32_t* n) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    const float2 y = __ffma2_rn(v, make_float2(r, r), make_float2(192.f, 192.f));
    const float2 z = __fadd2_rn(y, make_float2(kKv4Round, kKv4Round));
    n[2 * i] = __float_as_uint(z.x), n[2 * i + 1] = __float_as_uint(z.y);
  }
  if (careful) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
      n[i] = v != v ? 0x4b400000u + kKv4Zero : kv4_quantise(v, r);  // a NaN is held as zero
    }
  }
}

__device__ __forceinline__ uint32_t rot(uint32_t x, int b) { return b ? x << b | x >> (32 - b) : x; }

// A small append does in this launch what otherwise precedes it: it refreshes the block
// tables (a run a block, ahead of the pages' blocks) and copies the rows that a
// branch's first page takes over from a shared one.  Where another branch writes in place
// into that page, their words' other bits stay as they are.  Seven rows behind a fork,
// fork, append, read-back and release: 47 us with three launches, 44 with one.
template <int D>
__global__ void __launch_bounds__(2 * D) kv4_append_kernel(const Kv4StoreParams p,
                                                           const __grid_constant__ Kv4InlineAppend inl) {
  constexpr int kLanes = D / 8;       // threads of a row
  constexpr int kStride = D + 8;      // of the codes in shared memory: a page's two halves in different banks
  __shared__ __align__(8) uint8_t code_s[2][kPageTokens * kStride];
  griddep_wait();
  griddep_launch_dependents();
  const int layer = blockIdx.z;
  if ((int)blockIdx.x < p.n_table_blocks) {
    if (blockIdx.y || layer) return;
    const TableRun run = p.runs[blockIdx.x];
    for (int i = threadIdx.x; i < run.count; i += 2 * D) p.table_out[run.dst + i] = p.values[run.src + i];
    return;
  }
  const PageOfCall pg = page_of_call(p, p.branches ? p.branches : inl.b, blockIdx.x - p.n_table_blocks,
                                     p.small ? inl.pages : nullptr);
  // the page whose rows below `first` come into this one
  const int64_t from = p.small && pg.first > 0 ? inl.from[pg.branch] : -1;
  if ((uint64_t)pg.block >= (uint64_t)p.n_blocks || from >= p.n_blocks) {
    if (threadIdx.x == 0) atomicCAS(p.status, 0, kDevBadIndex);
    return;
  }
  const int t = threadIdx.x / kLanes, c = threadIdx.x % kLanes, g = c / 4;
  const int d = threadIdx.x / 2, h = threadIdx.x % 2;  // the word of V that this thread writes: 8 tokens of a channel
  const bool mine = t >= pg.first && t < pg.last, word = 8 * h < pg.last && 8 * h + 8 > pg.first;
  uint32_t ours = 0;  // the word's bits that are the call's
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (8 * h + i >= pg.first && 8 * h + i < pg.last) ours |= rot(15u, kv4_bit(i));
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  auto fetch = [&](int kvh) {
    if (!mine) return;
    const int64_t at = (((int64_t)layer * p.n_rows + pg.row + t) * p.Hkv + kvh) * D + c * 8;
    k = *reinterpret_cast<const uint4*>(p.k + at);
    v = *reinterpret_cast<const uint4*>(p.v + at);
  };
  fetch(blockIdx.y);
  if (!mine)  // tokens that are not the call's, in every head
#pragma unroll
    for (int b = 0; b < 2; ++b)
      *reinterpret_cast<uint2*>(code_s[b] + t * kStride + c * 8) = make_uint2(kKv4Zero * 0x01010101u, kKv4Zero * 0x01010101u);
  uint8_t* codes = code_s[0];
  for (int kvh = blockIdx.y; kvh < p.Hkv; kvh += gridDim.y) {
    const int64_t page = (((int64_t)layer * p.n_blocks + pg.block) * p.Hkv + kvh) * kv4_page_bytes(D);
    uint8_t* kp = p.k_pool + page;
    uint8_t* vp = p.v_pool + page;
    const int64_t back = from >= 0 ? (from - pg.block) * p.Hkv * kv4_page_bytes(D) : 0;  // to the rows taken over
    const uint4 kx = k, vx = v;
    if (kvh + (int)gridDim.y < p.Hkv) fetch(kvh + gridDim.y);  // on its way while this one is packed
    // of the group, four threads: two find the scale of its K and two that of its V
    const bool of_v = c & 1;
    uint32_t ka = max_bits8(kx), va = max_bits8(vx);
#pragma unroll
    for (int x = 1; x < 4; x *= 2) {
      ka = max(ka, __shfl_xor_sync(0xffffffffu, ka, x));
      va = max(va, __shfl_xor_sync(0xffffffffu, va, x));
    }
    float top = __uint_as_float((of_v ? va : ka) << 16);
    const bool careful = __any_sync(0xffffffffu, unusual(ka) || unusual(va));
    if (careful) {
      float kf = max_abs8(kx), vf = max_abs8(vx);
      for (int x = 1; x < 4; x *= 2) {
        kf = fmaxf(kf, __shfl_xor_sync(0xffffffffu, kf, x));
        vf = fmaxf(vf, __shfl_xor_sync(0xffffffffu, vf, x));
      }
      top = of_v ? vf : kf;
    }
    float scale;
    const uint32_t byte = kv4_make_scale(top, &scale);
    const float r = scale > 0.f ? __fdividef(1.f, scale) : 0.f;
    const float kr = __shfl_sync(0xffffffffu, r, threadIdx.x & 30), vr = __shfl_sync(0xffffffffu, r, threadIdx.x & 31 | 1);
    uint32_t n[8];
    if (mine) {
      codes8(kx, kr, careful, n);
      *reinterpret_cast<uint32_t*>(kp + g * 256 + t * 16 + (c & 3) * 4) = kv4_word(n);
      if ((c & 3) < 2) *((of_v ? vp + g * kPageTokens + t : kp + t * (D / kKv4Group) + g) + 8 * D) = (uint8_t)byte;
      codes8(vx, vr, careful, n);
      auto bytes = [&](int i) {
        return __byte_perm(__byte_perm(n[i], n[i + 1], 0x0040), __byte_perm(n[i + 2], n[i + 3], 0x0040), 0x5410);
      };
      *reinterpret_cast<uint2*>(codes + t * kStride + c * 8) = make_uint2(bytes(0), bytes(4));
    } else if (from >= 0 && t < pg.first) {
      const int at = g * 256 + t * 16 + (c & 3) * 4;
      *reinterpret_cast<uint32_t*>(kp + at) = *reinterpret_cast<const uint32_t*>(kp + back + at);
      if ((c & 3) == 0) {
        const int k_at = 8 * D + t * (D / kKv4Group) + g, v_at = 8 * D + g * kPageTokens + t;
        kp[k_at] = kp[back + k_at];
        vp[v_at] = vp[back + v_at];
      }
    }
    __syncthreads();  // a buffer is written again two heads later, behind the next of these
    if (word) {
      uint32_t* to = reinterpret_cast<uint32_t*>(vp + d * 8 + h * 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[i] = 0x4b400000u | codes[(8 * h + i) * kStride + d];
      }
      uint32_t w = kv4_word(n);
      if (~ours) w = (w & ours) | (*reinterpret_cast<const uint32_t*>(vp + back + d * 8 + h * 4) & ~ours);
      *to = w;
    } else if (from >= 0 && 8 * h < pg.first) {
      *reinterpret_cast<uint32_t*>(vp + d * 8 + h * 4) = *reinterpret_cast<const uint32_t*>(vp + back + d * 8 + h * 4);
    }
    codes = codes == code_s[0] ? code_s[1] : code_s[0];
  }
}

// Rows read back: a page as above; kKv4 false: of a bf16 pool.
template <int D, bool kKv4>
__global__ void __launch_bounds__(2 * D) read_kernel(const Kv4StoreParams p, const __grid_constant__ Kv4Branch rows) {
  constexpr int kLanes = D / 8;
  constexpr int kPageBytes = kKv4 ? kv4_page_bytes(D) : kPageTokens * D * 2;
  griddep_wait();
  griddep_launch_dependents();
  const int layer = blockIdx.z;
  const PageOfCall pg = page_of_call(p, &rows, blockIdx.x);
  if ((uint64_t)pg.block >= (uint64_t)p.n_blocks) {
    if (threadIdx.x == 0) atomicCAS(p.status, 0, kDevBadIndex);
    return;
  }
  const int t = threadIdx.x / kLanes, c = threadIdx.x % kLanes, g = c / 4;
  const bool mine = t >= pg.first && t < pg.last;
  auto page = [&](int kvh) { return (((int64_t)layer * p.n_blocks + pg.block) * p.Hkv + kvh) * kPageBytes; };
  auto row = [&](int kvh) { return (((int64_t)layer * p.n_rows + pg.row + t) * p.Hkv + kvh) * D + c * 8; };
  if constexpr (!kKv4) {
    if (!mine) return;
    for (int kvh = blockIdx.y; kvh < p.Hkv; kvh += gridDim.y) {
      const int64_t from = page(kvh) + (t * D + c * 8) * 2;
      *reinterpret_cast<uint4*>(p.k_out + row(kvh)) = *reinterpret_cast<const uint4*>(p.k_pool + from);
      *reinterpret_cast<uint4*>(p.v_out + row(kvh)) = *reinterpret_cast<const uint4*>(p.v_pool + from);
    }
  } else {
    // the page by way of shared memory, 8 channels of V every 72 bytes: a row's
    // threads then read their channels' words from different banks
    __shared__ __align__(16) uint8_t k_s[kPageBytes], v_s[9 * D], scales[D / 2];
    static_assert(kPageBytes / 8 <= 4 * D, "two pieces a thread");
    const int i = threadIdx.x;
    uint2 x[2];  // 8-byte pieces of K and V
    auto fetch = [&](int kvh) {
      if (i >= kPageBytes / 8) return;
      x[0] = *reinterpret_cast<const uint2*>(p.k_pool + page(kvh) + 8 * i);
      x[1] = *reinterpret_cast<const uint2*>(p.v_pool + page(kvh) + 8 * i);
    };
    fetch(blockIdx.y);
    for (int kvh = blockIdx.y; kvh < p.Hkv; kvh += gridDim.y) {
      if (i < kPageBytes / 8) {
        *reinterpret_cast<uint2*>(k_s + 8 * i) = x[0];
        *reinterpret_cast<uint2*>(i < D ? v_s + 8 * i + 8 * (i / 8) : scales + 8 * (i - D)) = x[1];
      }
      __syncthreads();
      if (kvh + (int)gridDim.y < p.Hkv) fetch(kvh + gridDim.y);
      if (mine) {
        const float ks = kv4_scale(k_s[8 * D + t * (D / kKv4Group) + g]), vs = kv4_scale(scales[g * kPageTokens + t]);
        const uint32_t kw = *reinterpret_cast<const uint32_t*>(k_s + g * 256 + t * 16 + (c & 3) * 4);
        uint32_t ko[4], vo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float kx[2], vx[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            kx[e] = kv4_code(kw, 2 * j + e) * ks;
            // token t % 8 is at the same place in every channel's word
            const uint32_t vw = *reinterpret_cast<const uint32_t*>(v_s + c * 72 + (2 * j + e) * 8 + (t >> 3) * 4);
            vx[e] = ((int)(__funnelshift_r(vw, vw, kv4_bit(t & 7)) & 15u) - 8) * vs;
          }
          const __nv_bfloat162 kk = __floats2bfloat162_rn(kx[0], kx[1]), vv = __floats2bfloat162_rn(vx[0], vx[1]);
          ko[j] = *reinterpret_cast<const uint32_t*>(&kk);
          vo[j] = *reinterpret_cast<const uint32_t*>(&vv);
        }
        *reinterpret_cast<uint4*>(p.k_out + row(kvh)) = make_uint4(ko[0], ko[1], ko[2], ko[3]);
        *reinterpret_cast<uint4*>(p.v_out + row(kvh)) = make_uint4(vo[0], vo[1], vo[2], vo[3]);
      }
      __syncthreads();
    }
  }
}

// Copy-on-write: whole pages (all KV heads of a layer lie together).  Rows past
// the copied ones come along; the sequence's own rows go over them.
__global__ void __launch_bounds__(256) kv4_copy_kernel(uint8_t* k_pool, uint8_t* v_pool, const CowCopy* cows,
                                                       const __grid_constant__ Kv4InlineCows inl, int64_t n_blocks,
                                                       int64_t page_bytes, int32_t* status) {
  griddep_wait();
  griddep_launch_dependents();
  const CowCopy c = cows ? cows[blockIdx.x] : inl.c[blockIdx.x];
  if ((uint64_t)c.src_block >= (uint64_t)n_blocks || (uint64_t)c.dst_block >= (uint64_t)n_blocks) {
    if (threadIdx.x == 0) atomicCAS(status, 0, kDevBadIndex);
    return;
  }
  const int64_t from = ((int64_t)blockIdx.y * n_blocks + c.src_block) * page_bytes;
  const int64_t to = ((int64_t)blockIdx.y * n_blocks + c.dst_block) * page_bytes;
  uint8_t* pool = blockIdx.z ? v_pool : k_pool;
  const uint4* src = reinterpret_cast<const uint4*>(pool + from);
  uint4* dst = reinterpret_cast<uint4*>(pool + to);
  for (int i = threadIdx.x; i < page_bytes / 16; i += blockDim.x) dst[i] = src[i];
}

// Blocks that share a page's heads: as many as fill the SMs some twice over.
int blocks_of_heads(const Kv4StoreParams& p) {
  const int64_t pages = (int64_t)p.n_pages * p.L, want = (2 * 152 * 8 + pages - 1) / pages;
  return (int)(want < p.Hkv ? want : p.Hkv);
}

}  // namespace

cudaError_t launch_kv4_append(const Kv4StoreParams& p, const Kv4InlineAppend* inl, int D, cudaStream_t s) {
  static const Kv4InlineAppend kNone{};
  if (p.n_pages == 0) return cudaSuccess;
  const dim3 grid(p.n_pages + p.n_table_blocks, blocks_of_heads(p), p.L);
  if (D == 128) return launch_chained(kv4_append_kernel<128>, grid, dim3(256), 0, s, p, inl ? *inl : kNone);
  if (D == 64) return launch_chained(kv4_append_kernel<64>, grid, dim3(128), 0, s, p, inl ? *inl : kNone);
  return cudaErrorInvalidValue;
}

cudaError_t launch_read_kv(const Kv4StoreParams& p, const Kv4Branch& rows, bool kv4, int D, cudaStream_t s) {
  if (p.n_pages == 0) return cudaSuccess;
  const dim3 grid(p.n_pages, blocks_of_heads(p), p.L);
  if (D == 128)
    return kv4 ? launch_chained(read_kernel<128, true>, grid, dim3(256), 0, s, p, rows)
               : launch_chained(read_kernel<128, false>, grid, dim3(256), 0, s, p, rows);
  if (D == 64)
    return kv4 ? launch_chained(read_kernel<64, true>, grid, dim3(128), 0, s, p, rows)
               : launch_chained(read_kernel<64, false>, grid, dim3(128), 0, s, p, rows);
  return cudaErrorInvalidValue;
}

cudaError_t launch_kv4_copy(uint8_t* k_pool, uint8_t* v_pool, const CowCopy* cows, const Kv4InlineCows* inl, int n,
                            int64_t n_blocks, int64_t page_bytes, int L, int32_t* status, cudaStream_t s) {
  static const Kv4InlineCows kNone{};
  if (n == 0) return cudaSuccess;
  return launch_chained(kv4_copy_kernel, dim3(n, L, 2), dim3(256), 0, s, k_pool, v_pool, cows, inl ? *inl : kNone,
                        n_blocks, page_bytes, status);
}

}  // namespace st
