// Pools that hold K and V in 4 bits (ST_FLAG_KV4): the format, and the
// parameter blocks and launchers of the kernels that write and read it.
//
// Values.  A row of a head is cut into groups of 32 values along D.  A group
// has a scale s = max |x| / 7, rounded to 4 significant bits (to even), in steps of
// at least 2^-17 and at most 3840; a value is held as n = x / s, rounded to even, within
// [-7, 7], and stands for n s.  The scale follows the group (4.25 bits a value in
// all), so that a channel that is larger than the others costs the precision of
// its 31 neighbours alone.  n has 3 significant bits and s has 4: n s is exact in
// bf16 and in f16, so what the attention multiplies is what the pool holds.
// N(0, 1) rows are off by 0.098 of their norm.
//
// Scale byte: the low 8 of (f16 bits of s) >> 7, that is 5 exponent and 3
// mantissa bits; s <= 3840 keeps 16.5 s, which the unpacking uses, in f16.
//
// A page of a head (16 tokens), K as V: 8 D bytes of codes, then D / 2 of scales,
// 17 D / 2 in all (1088 for D = 128), contiguous, a multiple of 32:
//   K  codes [D / 32][16 tokens][16 bytes]: a group of a token, dims 8 w ..
//      8 w + 7 in its w-th word; scales [16 tokens][D / 32]
//   V  codes [D][8 bytes]: a channel of the page's tokens, tokens 8 w .. 8 w + 7
//      in its w-th word; scales [D / 32][16 tokens]
// since the attention unpacks K by threads that have a token each and V by
// threads that have a channel each, into the two f16 of a 32-bit word that the
// tensor core reads along the dimension it sums over.
//
// A word has the codes n + 8 of 8 values v_0 .. v_7, v_{2 j} and v_{2 j + 1} at
// bits b_j and b_j + 16 (modulo 32), b = 6, 2, 14, 10: where the two f16 that the
// pair j becomes have the top four bits (j even) or the four below (j odd) of
// their mantissas, j = 2 and 3 after a rotation by 8.
#pragma once

#include <cuda_fp16.h>

#include "kernels.cuh"

namespace st {

constexpr int kKv4Group = 32;
constexpr float kKv4MaxScale = 3840.f;

// Bytes of a page of one head, of K or of V.
__host__ __device__ constexpr int kv4_page_bytes(int D) { return 17 * D / 2; }

// Where the codes of values 2 j and 2 j + 1 are in a word.
__host__ __device__ constexpr int kv4_bit(int i) { return ((0x0a0e0206 >> (8 * (i >> 1))) & 31) + 16 * (i & 1); }

// The code of value i of a word, in [-8, 7].
__device__ __forceinline__ int kv4_code(uint32_t w, int i) {
  const int b = kv4_bit(i);
  return (int)((w >> b | (b > 28 ? w << (32 - b) : 0u)) & 15u) - 8;
}

__device__ __forceinline__ float kv4_scale(uint32_t byte) {
  return __half2float(__ushort_as_half((unsigned short)(byte << 7)));
}

// The scale of a group whose largest magnitude is amax, as its byte and value.
__device__ __forceinline__ uint32_t kv4_make_scale(float amax, float* s) {
  const float x = fminf(__fdiv_rn(amax, 7.f), kKv4MaxScale);
  // from 2^-14 on 4 significant bits, rounded to even in the bits of x; steps of 2^-17 below
  const uint32_t u = __float_as_uint(x);
  float r = __uint_as_float((u + 0x7ffffu + ((u >> 20) & 1u)) & ~0xfffffu);
  if (x < 0x1p-14f) r = rintf(x * 0x1p17f) * 0x1p-17f;
  *s = r;
  return (uint32_t)__half_as_ushort(__float2half_rn(r)) >> 7;
}

// The code n of x under a scale with inverse r (0 for a scale of 0), as the bits of a
// float that end in kKv4Zero + n.  x r is off by 8 2^-22 (r by two of its last places), and x / s, a quotient of 8
// by 4 significant bits, is either in the middle between two codes or a
// thousandth away from it: rounded to steps of 2^-16 (where 192 + x r has its last
// place) it is in the middle exactly where x / s is, and the rounding to even that
// follows is that of x / s.  A NaN comes out as some code.
constexpr uint32_t kKv4Zero = 192;
constexpr float kKv4Round = 12582912.f;  // 1.5 2^23: rounds to whole numbers, and to even
__device__ __forceinline__ uint32_t kv4_quantise(float x, float r) {
  const float y = fmaxf(fminf(fmaf(x, r, 192.f), 199.f), 185.f);
  return __float_as_uint(y + kKv4Round);
}

// A word of eight codes, as kv4_quantise gives them.
__device__ __forceinline__ uint32_t kv4_word(const uint32_t* n) {
  uint32_t w = 0, bias = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (kv4_bit(i) > 28) continue;
    w += n[i] << kv4_bit(i);
    bias += 1u << kv4_bit(i);
  }
  // value 5 is at bits 30, 31, 0 and 1
  static_assert(kv4_bit(5) == 30, "the value that wraps");
  const uint32_t five = (n[5] & 255u) - (kKv4Zero - 8);
  return w - bias * (0x4b400000u + kKv4Zero - 8) + (five << 30 | five >> 2);
}

// Rows of a sequence at most: their numbers are 32 bits wide here, up to the end of the
// last stage of keys.  (A bf16 pool's memory ends before that.)
constexpr int64_t kKv4MostRows = INT32_MAX - 255;

// ---- append, copy, read back (kv4_store.cu) --------------------------------------

struct Kv4Branch {
  int32_t slot;
  int32_t start;  // sequence length before this call
  int32_t row0;   // first of this branch's rows in the call's input
  int32_t n;      // rows
  int32_t page0;  // pages of the branches before it
};
struct Kv4StoreParams {
  const __nv_bfloat16* k;  // [L][n_rows][Hkv][D]
  const __nv_bfloat16* v;
  __nv_bfloat16* k_out;    // read back: the same shape
  __nv_bfloat16* v_out;
  uint8_t* k_pool;         // [L][n_blocks][Hkv][page bytes] (bf16 pages, in a read of a bf16 pool)
  uint8_t* v_pool;
  const int32_t* table;    // [max_seqs][max_pages]
  const Kv4Branch* branches;  // null: in the inline block
  int32_t* status;
  int64_t n_blocks;
  int32_t n_br, n_rows, n_pages, L, Hkv, max_pages;  // n_pages: of all branches
  // a small append: pages and copies in the inline block, the tables refreshed in blocks of this launch
  int32_t small, n_table_blocks;
  int32_t* table_out;
  const TableRun* runs;
  const int32_t* values;
};

// Pages of a small append in the order of its branches, and (or -1) the page whose rows
// below a branch's first one come into its first page.
struct Kv4InlineAppend {
  Kv4Branch b[kInlineAppendBranches];
  int32_t from[kInlineAppendBranches];
  int32_t pages[kInlinePages];
};
constexpr int kKv4TableBlocks = 32;  // most of a small append

cudaError_t launch_kv4_append(const Kv4StoreParams& p, const Kv4InlineAppend* inl, int D, cudaStream_t s);
// Rows of one branch read back, from a 4-bit pool or (kv4 false) a bf16 one.
cudaError_t launch_read_kv(const Kv4StoreParams& p, const Kv4Branch& rows, bool kv4, int D, cudaStream_t s);

struct Kv4InlineCows {
  CowCopy c[kInlineCows];
};
// Whole pages of every layer; cows null: in the inline block.
cudaError_t launch_kv4_copy(uint8_t* k_pool, uint8_t* v_pool, const CowCopy* cows, const Kv4InlineCows* inl, int n,
                            int64_t n_blocks, int64_t page_bytes, int L, int32_t* status, cudaStream_t s);

// ---- attention (kv4_attend.cu) ------------------------------------------------------

constexpr int kKv4Rows = 64;  // stacked query rows of a tile; twice as many of a wide one
constexpr int kKv4Keys = 128; // keys of a stage

// A tile of a prefill: 64 (wide: 128) stacked (new row, head) rows from row_base on
// of one sequence over the keys of pages [page_begin, page_begin + n_pages).
struct Kv4Tile {
  int32_t slot;
  int32_t L0;       // the sequence's length before this call
  int32_t T;        // rows appended to it
  int32_t q_row0;   // its first row in the call's Q
  int32_t row_base;
  int32_t page_begin, n_pages;
  int32_t split;    // partial slot; -1: the tile sees all its keys, O and LSE are final
};

struct Kv4AttnParams {
  const __nv_bfloat16* q;   // [L][n_rows_q][Hq][D]
  const uint8_t* k_pool;
  const uint8_t* v_pool;
  float* part_o;            // [L][n_rows_q][Hq][max_splits][D]
  float* part_lse;
  __nv_bfloat16* o;         // final results of a prefill
  float* lse;
  const int32_t* table;
  const AttnItem* items;    // decode; null: in the inline plan
  const int32_t* members;
  const Kv4Tile* tiles;     // prefill
  int32_t* status;
  int64_t n_blocks;
  float scale_log2;         // log2(e) / sqrt(D)
  int32_t n_items, n_rows_q, Hq, Hkv, G, L, max_pages, max_splits;
  int32_t hold_loads;       // test hook (ST_FLAG_HOLD_LOADS)
  int32_t wide;             // works of up to 128 rows
  int32_t keep_l2;          // pages are loaded to stay in L2: a decode's that fit there, a prefill's, which several row tiles read
};

cudaError_t launch_kv4_attend(const Kv4AttnParams& p, const InlineDecodePlan* inl, int D, cudaStream_t s);

// The combine of combine.cu with O in bf16.  uniform: partials of every row (0: p.n_splits, or the inline counts).
cudaError_t launch_combine_bf16(const CombineParams& p, const InlineSplits* inl, __nv_bfloat16* o, int uniform, int D,
                                cudaStream_t s);

}  // namespace st
