// Attention over a pool that holds K and V in 4 bits (format: kv4.cuh), on the
// 5th-generation tensor cores: decode partials of stacked query rows over a run of
// pages, and causal prefill tiles.
//
// A 4-bit page is a quarter of a bf16 one, so unpacking it must not cost what
// reading it saves.  Unpacked rows written to shared memory and read from there by
// the tensor core would move 3.8 bytes twice for each byte that comes in, more
// than an SM's shared memory passes at the rate HBM delivers.  So the products
// are taken with K and V on the left, where the tensor core reads its operand from
// tensor memory, and the unpacked values go there straight from registers:
//   S^T = K Q^T     [128 keys x rows]   A: K, a key in a lane, D / 2 columns
//   O^T += V^T P^T  [D x rows]          A: V, a channel in a lane, 64 columns
// with Q and P, which are small, on the right in shared memory.  Both operands
// are f16: n s / 16 is exact in it, the queries are scaled by a power of two to the top of
// its range and the scores back in 32 bits, and P is rounded to it, 2^-11 of each weight where
// O is rounded to 2^-8 at the end.  A work's rows have one power of two where their largest
// values are within 2^8 of each other (a row is then off by 2^-30 of its largest value at
// most, against 2^-23 of each sum), and else each its own, so that no row's result depends
// on another's size: their scores are then rescaled where they lie, in a copy of the
// softmax, which a pass over like rows does not run (looking which it is costs 1 to 2%; with a
// scale of its own for every row of every work 24 branches took 348 us against 308).  Sums,
// maxima, statistics and O are in 32 bits.
//
// A block (one an SM, 20 warps) takes work after work, a work being a run of pages
// (or a prefill tile) of one KV head and layer for up to 64 rows.  Its stages of
// 128 keys go in turn to two streams, each with K, V, S, P and O of its own, so
// that every step of a stage has the time of two, and what a stage costs a warp
// besides its values (waits, addresses) is paid by 4 warps and not by 8.
//
// A wide work has up to 128 rows: those of a group beyond 64, and of a prefill.  Each softmax
// group then takes every stage, for half of the rows, and the two share a stage's K and
// V, which lie in the stages' two places in turn.  What is unpacked once serves twice the
// rows: 24 branches of 8 heads over 65536 tokens, two groups and layers, 396 -> 364 us (315 since, with
// longer runs and rows by eights); 2048 rows of 32/8 heads onto 16896, four layers, 3340 -> 2980 (2810
// since, with registers shared out for it).  Roles:
//   0..7    softmax, two groups of 128 threads: thread t has key t of
//           a stage, a score of each row.  The reference of a row is 8 (log2)
//           below the maximum when it was last set, and set anew only when a score
//           comes 15 above it, 7 above that maximum (f16 holds 2^16): then the
//           group finds the new maximum and rescales its O and sums.  Scores so large that
//           fp32 has them off by more than that count as at most 15 above.  Sums stay
//           per key until the work's end, where a narrow work's two streams are joined.
//   8..15   unpacking, a group for every other stage: thread t unpacks key t of K, then
//           channel t of V (a group's 32 channels are one warp's, so that a token's
//           scale is one for the warp) into tensor memory
//   16      loader: 8 pages of K and V a stage, 16 bulk copies
//   17, 18  tensor core instructions of a softmax group, S of a stage ahead of the P V
//           before it.  A warp for each, since one that serves both in
//           turn holds either back until the other is ready.  The whole warp
//           runs the loop, with operands that are the same for all lanes, and one
//           elected lane issues: 24 cycles an instruction of 48 rows, where one lane
//           that runs alone takes over 100
//   19      the queries of the next work
//
// What bounds it: the latencies of these roles.  A stage of 40 rows takes a block 1500 cycles (131072
// tokens of 5 branches, four agents and layers: 3.2 TB/s of pages), one of 128 rows 2500;
// the tensor core is busy for some 400 and 1050 of them, the exponentials take 320 and 1000 of
// their pipe, instructions go out in half of the cycles, and the loads would come at
// 5.6 TB/s.  The unpacking groups have the least slack: a stream's stage takes 3400 cycles, its
// K and V some 3070 of their group, a softmax group's part 2230.
//
// How far sums reach: the tensor core cuts off each step of O's, so over equal weights of one
// sign O is low by 1e-4 of itself at 2^20 keys a run, 2e-3 at 2^22, 8e-3 at 2^23.
#include <math.h>

#include <mutex>

#include "kv4.cuh"
#include "ptx.cuh"

namespace st {

namespace {

constexpr int kThreads = 640;
constexpr int kUnpackWarp = 8, kLoadWarp = 16, kMmaWarp = 17, kQWarp = 19;
constexpr int kPages = kKv4Keys / kPageTokens;  // of a stage
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kTmemK = 0, kTmemV = 128, kTmemS = 256, kTmemO = 384;  // 64 columns for each of two
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kUnset = -1e30f;      // a row's reference before it has seen a key: finite, any will do
constexpr float kHeadroom = 15.f, kBelow = 8.f;
constexpr float kOff = 0x1p-21f;      // of a score and its reference: eight roundings
constexpr int kAlike = 8;             // powers of two between rows that have one scale
constexpr int kMaxDevices = 64;
// Registers a thread: what the block is launched with is shared out anew among its
// five warpgroups (the softmax has a sum, and up to 64 rows a score, of each row in
// them).  setmaxnreg.inc waits without a limit for registers that the block does not
// have, so a build that launches with fewer is refused.
constexpr int kLaunchRegs = 96;
// A wide prefill's groups have 64 rows each as a rule, and with 144 registers wait for what
// they spilled (four layers, 2048 rows onto 16896, in a short run: 2.98 ms against 2.56 with 160;
// with 152 2.99, with 168 2.74); a decode's have fewer, and unpacking with 56 costs it 8% (24 branches).
template <bool kCausal, bool kWide>
struct Regs {
  static constexpr bool kMore = kCausal && kWide;
  static constexpr int kSoft = kMore ? 160 : 144, kUnpack = kMore ? 56 : 64, kAux = kMore ? 48 : 64;
  static constexpr bool suffice(int launch) {
    return 5 * launch >= 2 * kSoft + 2 * kUnpack + kAux && launch >= kUnpack && launch <= kSoft;
  }
  static_assert(suffice(kLaunchRegs) && !suffice(kLaunchRegs - 1), "registers of a block");
};

template <int D, bool kWide>
struct Cfg {
  static constexpr int kPage = kv4_page_bytes(D);
  static constexpr int kStageBytes = 2 * kPages * kPage;
  static constexpr int kStages = D == 128 ? 6 : 10;
  static constexpr int kQTile = (D / 64) * kKv4Rows * 128;
  static constexpr int kQBytes = kWide ? 2 * kQTile : kQTile;  // a buffer
  static constexpr int kPBytes = kKv4Keys * 128;
  static constexpr int kOffP = 2 * kQBytes;
  static constexpr int kOffRing = kOffP + 2 * kPBytes;
  static constexpr int kOffScales = kOffRing + kStages * kStageBytes;  // V scales, 512 bytes a warp
  static constexpr int kOffMeta = kOffScales + 8 * 512;
  static constexpr int kSmemBytes = kOffMeta + 8192 + 1024;            // 1024: to align it
};

// Rows and state that roles share, for two works.
struct Meta {
  float m[2][kKv4Rows];       // of each group: references, negative
  float f[2][kKv4Rows];       // factors of O
  float sum[2][kKv4Rows];     // sums at a work's end
  int32_t red[2][4][kKv4Rows];
  int64_t row[2][2 * kKv4Rows];   // row of Q (layer, row, head), -1 beyond the work's
  int32_t seen[2][2 * kKv4Rows];  // prefill: keys of the run that the row sees
  float own[2][2 * kKv4Rows];     // unlike rows: a row's own share of the scale, negative
  float scale[2];             // of the scores, log2 domain; negative where the rows are unlike
  uint32_t tmem;
  uint64_t bars[52];
};
static_assert(sizeof(Meta) <= 8192, "meta area");

struct Work {
  int slot, page0, n_pages, n_keys, n_rows, kvh, layer, split;
  int member_base;          // decode
  int L0, q_row0, row_base; // prefill
};

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
          smem_addr(dst)),
      "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(smem_addr(bar)), "l"(policy)
      : "memory");
}

// 16 bytes to shared memory, or zeros.
__device__ __forceinline__ void copy16_async(void* dst, const void* src, bool has) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)),
               "l"(__cvta_generic_to_global(src)), "r"(has ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// This warpgroup's registers a thread, out of those that each was launched with.
template <int N>
__device__ __forceinline__ void set_registers() {
  if constexpr (N > kLaunchRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// Barrier `id` of kN threads; true where the predicate holds for any.
template <int kN>
__device__ __forceinline__ bool any_of(int id, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(id), "n"(kN)
      : "memory");
  return r != 0;
}

// One lane of the (converged) warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* v) {
  uint32_t r[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// N columns of this thread's lane, a multiple of 8 from 16 to 64.
template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, float* v) {
  if constexpr (N >= 32) {
    tmem_ld32(taddr, v);
    if constexpr (N == 64) tmem_ld32(taddr + 32, v + 32);
    else if constexpr (N >= 48) tmem_ld16(taddr + 32, v + 32);
    if constexpr (N % 16) tmem_ld8(taddr + N - 8, v + N - 8);
  } else {
    tmem_ld16(taddr, v);
    if constexpr (N == 24) tmem_ld8(taddr + 16, v + 16);
  }
}

__device__ __forceinline__ void tmem_st8u_nowait(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]),
               "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

__device__ __forceinline__ constexpr uint32_t idesc_f16(int N) {  // f16 in, fp32 out, M = 128, B as given below
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
}
constexpr uint32_t kIdescBMnMajor = 1u << 16;

// A value that all lanes have, as one that the compiler knows to be the warp's: loops
// and operands made of such values stay in uniform registers, from which the
// instructions of the tensor core and of the bulk copies take them.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_max_sync(0xffffffffu, x); }

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }

// (w & mask) | exponent as two f16, in one instruction (the operators take two, and
// this half-rate pipe is the fullest).
__device__ __forceinline__ __half2 bits_under(uint32_t w, uint32_t mask, uint32_t exponent) {
  uint32_t x;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w), "r"(mask), "r"(exponent));
  return as_half2(x);
}

// The 8 values of a word over 16, as four pairs.  With the code's bits at the top
// of a mantissa the f16 is 1 + n' / 16 (n' = n + 8) or, four bits lower under 2^4, 16 + n' / 16;
// times s, less 1.5 s or 16.5 s, both exact, in one fused step that is exact too.
// s: the scale of each pair; c: -1.5 s (pairs 0 and 2) or -16.5 s (1 and 3).
__device__ __forceinline__ void unpack8(uint32_t w, const uint32_t* s, const uint32_t* c, uint32_t* out) {
  const uint32_t r = __funnelshift_r(w, w, 8);
  out[0] = as_u32(__hfma2(bits_under(w, 0x03c003c0u, 0x3c003c00u), as_half2(s[0]), as_half2(c[0])));
  out[1] = as_u32(__hfma2(bits_under(w, 0x003c003cu, 0x4c004c00u), as_half2(s[1]), as_half2(c[1])));
  out[2] = as_u32(__hfma2(bits_under(r, 0x03c003c0u, 0x3c003c00u), as_half2(s[2]), as_half2(c[2])));
  out[3] = as_u32(__hfma2(bits_under(r, 0x003c003cu, 0x4c004c00u), as_half2(s[3]), as_half2(c[3])));
}

__device__ __forceinline__ uint32_t scaled(uint32_t s, float by) {
  return as_u32(__hmul2(as_half2(s), __float2half2_rn(by)));
}

template <int D, bool kCausal, bool kWide>
struct Kernel {
  using C = Cfg<D, kWide>;
  static constexpr int kStep = kWide ? 1 : 2;  // from a stage of a softmax group to its next
  const Kv4AttnParams& p;
  const InlineDecodePlan& inl;
  uint8_t* base;
  Meta& meta;
  uint32_t tmem;
  int n_works;

  uint64_t *raw_full, *raw_empty, *k_full, *k_empty, *v_full, *v_empty, *pv_done, *s_full, *s_empty, *p_full, *q_full, *q_empty,
      *o_empty;

  __device__ __forceinline__ Kernel(const Kv4AttnParams& params, const InlineDecodePlan& plan, uint8_t* b)
      : p(params), inl(plan), base(b), meta(*reinterpret_cast<Meta*>(b + C::kOffMeta)) {
    n_works = p.n_items * p.Hkv * p.L;
    uint64_t* at = meta.bars;
    auto take = [&](int n) {
      uint64_t* r = at;
      at += n;
      return r;
    };
    raw_full = take(C::kStages), raw_empty = take(C::kStages);
    k_full = take(2), k_empty = take(2), v_full = take(2), pv_done = take(2), s_full = take(2), s_empty = take(2);
    p_full = take(2), q_full = take(2), q_empty = take(2), o_empty = take(2);
    v_empty = kWide ? take(2) : pv_done;
    static_assert(2 * C::kStages + 24 <= 52, "barriers");
  }

  __device__ __forceinline__ void init_barriers() {
    for (int i = 0; i < C::kStages; ++i) mbar_init(&raw_full[i], 1), mbar_init(&raw_empty[i], 4);
    for (int b = 0; b < 2; ++b) {
      mbar_init(&k_full[b], 4);
      mbar_init(&k_empty[b], kWide ? 2 : 1);
      if (kWide) mbar_init(&v_empty[b], 2);
      mbar_init(&v_full[b], 4);
      mbar_init(&pv_done[b], 1);
      mbar_init(&s_full[b], 1);
      mbar_init(&s_empty[b], 4);
      mbar_init(&p_full[b], 4);
      mbar_init(&q_full[b], 1);
      mbar_init(&q_empty[b], 10);
      mbar_init(&o_empty[b], kWide ? 4 : 8);
    }
    fence_mbar_init();
  }

  __device__ __forceinline__ Work work_at(int w) const {
    const int per = p.Hkv * p.L, i = w / per, rest = w % per;
    Work k;
    k.kvh = rest % p.Hkv;
    k.layer = rest / p.Hkv;
    if constexpr (kCausal) {
      const Kv4Tile t = p.tiles[i];
      k.slot = t.slot, k.page0 = t.page_begin, k.n_pages = t.n_pages, k.split = t.split;
      k.L0 = t.L0, k.q_row0 = t.q_row0, k.row_base = t.row_base;
      k.n_rows = (int)min((int64_t)(kWide ? 2 : 1) * kKv4Rows, (int64_t)t.T * p.G - t.row_base);
      k.n_keys = min(t.n_pages * kPageTokens, t.L0 + t.T - t.page_begin * kPageTokens);
    } else {
      const AttnItem t = p.items ? p.items[i] : inl.items[i];
      k.slot = t.slot, k.page0 = t.page_begin, k.n_pages = t.n_pages, k.split = t.split;
      k.member_base = t.member_base;
      k.n_rows = t.n_members * p.G;
      k.n_keys = t.n_tokens;
    }
    return k;
  }
  // The work after the n-th, w, of this block.  Works come longest first, and every other
  // round of the blocks goes backwards, so that a block's are long and short.
  __device__ __forceinline__ static int after(int w, int n) { return (2 * n + 2) * (int)gridDim.x - 1 - w; }
  __device__ __forceinline__ static int stages_of(const Work& k) { return (k.n_pages + kPages - 1) / kPages; }
  // A softmax group's rows, with those that fill it up (the rest of a wide work's are the other's).
  __device__ __forceinline__ static int cols_of(const Work& k) {
    return ((kWide ? (k.n_rows + 1) / 2 : k.n_rows) + 15) / 16 * 16;
  }
  // The stage g of a block: its turn among those of a softmax group, and among those of its place of K and V.
  __device__ __forceinline__ static uint32_t turn(int g) { return (kWide ? g : g >> 1) & 1; }
  __device__ __forceinline__ static uint32_t place_turn(int g) { return g >> 1 & 1; }

  // Every lane waits; true where all have seen the phase end.
  __device__ __forceinline__ static bool wait(uint64_t* bar, uint32_t parity) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "vote.sync.all.pred q, p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    if (all) return true;
    return __all_sync(0xffffffffu, mbar_wait(bar, parity));
  }
  // Whether the phase has ended, without a wait (try_wait may suspend the thread until it has).
  __device__ __forceinline__ static bool ended(uint64_t* bar, uint32_t parity) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "vote.sync.all.pred q, p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return all != 0;
  }
  struct Slot {  // of the ring of stages
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() {
      if (++s == C::kStages) s = 0, parity ^= 1;
    }
  };
  __device__ __forceinline__ void timeout(bool ok, int lane) {
    if (!ok && lane == 0) atomicCAS(p.status, 0, kDevTimeout);
  }

  // ---- loader ------------------------------------------------------------------
  __device__ __forceinline__ void load(int lane) {
    if (p.hold_loads) return;  // test hook: nothing arrives, the other roles' waits run out
    const uint64_t policy = p.keep_l2 ? l2_policy_evict_normal() : l2_policy_evict_first();
    const int page_stride = p.Hkv * C::kPage;
    int g = 0;
    Slot slot;
    bool ok = true;
    for (int w = blockIdx.x, n = 0; ok && w < n_works; w = after(w, n++)) {
      const Work k = work_at(w);
      const int32_t* ids = p.table + (int64_t)k.slot * p.max_pages + k.page0;
      const int stages = (int)uniform(stages_of(k)), n_pages = (int)uniform(k.n_pages);
      const int64_t head = ((int64_t)k.layer * p.n_blocks * p.Hkv + k.kvh) * C::kPage;
      const uint8_t* kb = p.k_pool + head;
      const uint8_t* vb = p.v_pool + head;
      // page ids, 32 at a time (four stages), the next ones on their way
      int cur = lane < n_pages ? ids[lane] : 0, nxt = 32 + lane < n_pages ? ids[32 + lane] : 0;
      for (int t = 0; t < stages; ++t, ++g, slot.next()) {
        if (t > 0 && t % 4 == 0) {
          cur = nxt;
          const int page = t * kPages + 32 + lane;
          nxt = page < n_pages ? ids[page] : 0;
        }
        if ((uint64_t)cur >= (uint64_t)p.n_blocks) {
          atomicCAS(p.status, 0, kDevBadIndex);
          cur = 0;
        }
        const int np = min(kPages, n_pages - t * kPages);
        int block[kPages];
#pragma unroll
        for (int q = 0; q < kPages; ++q) block[q] = __shfl_sync(0xffffffffu, cur, t % 4 * kPages + q);
        if (!(ok = wait(&raw_empty[slot.s], slot.parity ^ 1))) break;
        uint8_t* to = base + C::kOffRing + slot.s * C::kStageBytes;
        uint64_t* bar = &raw_full[slot.s];
        if (elect_one()) {
          mbar_arrive_expect_tx(bar, 2 * np * C::kPage);
#pragma unroll
          for (int q = 0; q < kPages; ++q) {
            if (q < np) {
              const int64_t at = (int64_t)block[q] * page_stride;
              bulk_load(to + q * C::kPage, kb + at, C::kPage, bar, policy);
              bulk_load(to + (kPages + q) * C::kPage, vb + at, C::kPage, bar, policy);
            }
          }
        }
        __syncwarp();
      }
    }
    timeout(ok, lane);
    if (!ok)  // copies in flight land before the block ends
      for (int i = max(0, g - C::kStages); i < g; ++i) wait(&raw_full[i % C::kStages], i / C::kStages & 1);
  }

  // ---- unpacking: a key of K, or a channel of V a thread ------------------------------
  // A stream's stages, over the works.
  struct Cursor {
    int w, n, t, stages, n_keys;
    Slot slot;
    uint32_t parity;  // of the stage before, among the stream's
  };
  __device__ __forceinline__ void settle(Cursor* c) const {  // t may lie in a later work
    while (c->w < n_works && c->t >= c->stages) {
      c->t -= c->stages;
      c->w = after(c->w, c->n++);
      if (c->w >= n_works) break;
      const Work k = work_at(c->w);
      c->stages = stages_of(k);
      c->n_keys = k.n_keys;
    }
  }
  __device__ __forceinline__ Cursor first_stage(int stream) const {
    Cursor c{(int)blockIdx.x, 0, stream, 0, 0, Slot(), 1};
    if (c.w < n_works) {
      const Work k = work_at(c.w);
      c.stages = stages_of(k);
      c.n_keys = k.n_keys;
    }
    if (stream) c.slot.next();
    settle(&c);
    return c;
  }
  __device__ __forceinline__ void advance(Cursor* c) const {
    c->t += 2;
    c->slot.next();
    c->slot.next();
    c->parity ^= 1;
    settle(c);
  }

  __device__ __forceinline__ bool unpack_k(const Cursor& at, int stream, int warp, int lane) {
    const int key = warp * 32 + lane, tok = key % kPageTokens;
    if (!wait(&raw_full[at.slot.s], at.slot.parity)) return false;
    const uint8_t* page = base + C::kOffRing + at.slot.s * C::kStageBytes + key / kPageTokens * C::kPage;
    uint4 code[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c) code[c] = *reinterpret_cast<const uint4*>(page + c * 256 + tok * 16);
    uint32_t scales;
    if constexpr (D == 128) scales = *reinterpret_cast<const uint32_t*>(page + 8 * D + tok * 4);
    else scales = *reinterpret_cast<const uint16_t*>(page + 8 * D + tok * 2);
    if (!wait(&k_empty[stream], at.parity)) return false;
    tc_fence_after_sync();
    const uint32_t to = tmem + ((uint32_t)(warp * 32) << 16) + kTmemK + stream * 64;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const uint32_t one = (scales >> (8 * c) & 255u) << 7;
      const uint32_t s2 = one | one << 16;
      const uint32_t sc[4] = {s2, s2, s2, s2};
      const uint32_t hi = scaled(s2, -1.5f), lo = scaled(s2, -16.5f);
      const uint32_t cc[4] = {hi, lo, hi, lo};
      uint32_t out[16];
      unpack8(code[c].x, sc, cc, out);
      unpack8(code[c].y, sc, cc, out + 4);
      unpack8(code[c].z, sc, cc, out + 8);
      unpack8(code[c].w, sc, cc, out + 12);
      tmem_st16u_nowait(to + c * 16, out);
    }
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&k_full[stream]);
    return true;
  }

  // The stage's K has been unpacked, so its pages have landed.
  __device__ __forceinline__ bool unpack_v(const Cursor& at, int stream, int warp, int lane) {
    const int d = warp * 32 + lane;
    const bool live = warp < D / 32;
    // scales and offsets, 4 tokens each
    uint4* table = reinterpret_cast<uint4*>(base + C::kOffScales + (stream * 4 + warp) * 512);
    const uint8_t* stage = base + C::kOffRing + at.slot.s * C::kStageBytes + kPages * C::kPage;
    if (live) {
      const uint32_t four = *reinterpret_cast<const uint32_t*>(stage + lane / 4 * C::kPage + 8 * D +
                                                               warp * kPageTokens + lane % 4 * 4);
      uint32_t sa = (four & 0xffu) << 7 | (four & 0xff00u) << 15;
      uint32_t sb = (four & 0xff0000u) >> 9 | (four & 0xff000000u) >> 1;
      // tokens past the run, and pages that were not loaded: what lies there
      // (it may be no number) counts for nothing
      const int left = at.n_keys - at.t * kKv4Keys - lane * 4;
      if (left < 4) {
        sa &= (left > 0 ? 0xffffu : 0u) | (left > 1 ? 0xffff0000u : 0u);
        sb &= left > 2 ? 0xffffu : 0u;
      }
      table[lane] = make_uint4(sa, scaled(sa, -1.5f), sb, scaled(sb, -16.5f));
      __syncwarp();
    }
    if (!wait(&v_empty[stream], at.parity)) return false;
    tc_fence_after_sync();
    if (live) {
      const uint32_t to = tmem + ((uint32_t)(warp * 32) << 16) + kTmemV + stream * 64;
#pragma unroll 1
      for (int q = 0; q < kPages; q += 2) {
        uint32_t out[16];
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // pages, two words of 8 tokens each
          const uint2 word = *reinterpret_cast<const uint2*>(stage + (q + i) * C::kPage + d * 8);
          const uint4* x = table + (q + i) * 4;
          const uint4 a = x[0], b = x[1], c = x[2], e = x[3];
          const uint32_t s0[4] = {a.x, a.z, b.x, b.z}, c0[4] = {a.y, a.w, b.y, b.w};
          const uint32_t s1[4] = {c.x, c.z, e.x, e.z}, c1[4] = {c.y, c.w, e.y, e.w};
          unpack8(word.x, s0, c0, out + 8 * i);
          unpack8(word.y, s1, c1, out + 8 * i + 4);
        }
        tmem_st16u_nowait(to + q * 8, out);
      }
      tmem_wait_st();
    }
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(&raw_empty[at.slot.s]);
      mbar_arrive(&v_full[stream]);
    }
    return true;
  }

  // K a stage ahead of V, whose place is free only when the product before has read it.
  __device__ __forceinline__ void unpack(int stream, int warp, int lane) {
    Cursor k = first_stage(stream), v = k;
    bool ok = k.w >= n_works || unpack_k(k, stream, warp, lane);
    if (k.w < n_works) advance(&k);
    while (ok && v.w < n_works) {
      if (k.w < n_works) {
        ok = unpack_k(k, stream, warp, lane);
        advance(&k);
      }
      ok = ok && unpack_v(v, stream, warp, lane);
      advance(&v);
    }
    timeout(ok, lane);
  }

  // ---- tensor core instructions -------------------------------------------------------
  __device__ __forceinline__ void issue(int which, int lane) {
    const int group = (int)uniform(which);
    const uint64_t q_desc = tc_desc_sw128(smem_addr(base + (kWide ? group * C::kQTile : 0)), 16, 1024);
    const uint64_t p_desc = tc_desc_sw128(smem_addr(base + C::kOffP + group * C::kPBytes), 16, 1024);
    const uint32_t at = uniform(tmem);
    const uint32_t s_at = at + kTmemS + group * 64, o_at = at + kTmemO + group * 64;
    bool ok = true, pending = false;      // whether a stage's P V is still to be issued
    int pv_n = 0, pv_cols = 0, pv_g = 0;  // its work, rows and stage of the block
    bool pv_first = false;                // and whether it is the first of its group in its work
    auto issue_pv = [&]() -> bool {
      const int place = kWide ? pv_g & 1 : group;
      if (!wait(&p_full[group], turn(pv_g)) || !wait(&v_full[place], place_turn(pv_g))) return false;
      if (pv_first && pv_n > 0 && !wait(&o_empty[kWide ? group : 0], (pv_n - 1) & 1)) return false;
      tc_fence_after_sync();
      const uint32_t idesc = idesc_f16(pv_cols) | kIdescBMnMajor, v_at = at + kTmemV + place * 64;
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < kKv4Keys / 16; ++kk)
          tc_mma_bf16_tmem_a(o_at, v_at + kk * 8, p_desc + (uint64_t)((kk * 2048) >> 4), idesc, kk > 0 || !pv_first);
        tc_commit(&pv_done[group]);
        if (kWide) tc_commit(&v_empty[place]);
      }
      __syncwarp();
      pending = false;
      return true;
    };
    int g0 = 0, n = 0;
    for (int w = blockIdx.x; ok && w < n_works; w = after(w, n++)) {
      const Work k = work_at(w);
      const int stages = (int)uniform(stages_of(k)), cols = (int)uniform(cols_of(k));
      const uint32_t idesc = idesc_f16(cols);
      const uint64_t qd = q_desc + (uint64_t)(((n & 1) * C::kQBytes) >> 4);
      const int t0 = kWide ? 0 : (g0 ^ group) & 1;
      // a P V does not wait for queries
      if (pending && !ended(&q_full[n & 1], n >> 1 & 1) && !(ok = issue_pv())) break;
      if (!(ok = wait(&q_full[n & 1], n >> 1 & 1))) break;
      // a stream without a stage here has read the queries as far as it ever will
      if (t0 >= stages && lane == 0) mbar_arrive(&q_empty[n & 1]);
      for (int t = t0; t < stages; t += kStep) {
        const int g = g0 + t, place = kWide ? g & 1 : group;
        if (!(ok = wait(&k_full[place], place_turn(g)) && wait(&s_empty[group], turn(g) ^ 1))) break;
        tc_fence_after_sync();
        if (elect_one()) {
          const uint32_t k_at = at + kTmemK + place * 64;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            tc_mma_bf16_tmem_a(s_at, k_at + kk * 8,
                               qd + (uint64_t)(((kk >> 2) * kKv4Rows * 128 + (kk & 3) * 32) >> 4), idesc, kk != 0);
          tc_commit(&s_full[group]);
          tc_commit(&k_empty[place]);
          if (t + kStep >= stages) tc_commit(&q_empty[n & 1]);
        }
        __syncwarp();
        if (pending && !(ok = issue_pv())) break;
        pv_n = n, pv_cols = cols, pv_g = g, pv_first = t < kStep, pending = true;
      }
      g0 += stages;
    }
    if (ok && pending) ok = issue_pv();
    timeout(ok, lane);
    if (!ok) {  // what was issued is through before tensor memory is freed
      const unsigned long long t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 1000000ull) {}
    }
  }

  // ---- queries ------------------------------------------------------------------------
  __device__ __forceinline__ void queries(int lane) {
    constexpr int kChunks = D / 8;  // of 16 bytes in a row
    int n = 0;
    bool ok = true;
    int ahead[2] = {0, 0};  // stages of the works whose queries a buffer has
    for (int w = blockIdx.x; w < n_works; w = after(w, n++)) {
      const int b = n & 1;
      // the one wait for a whole work, which may take longer than a wait's limit: another for each 2^18 stages
      const int waits = 1 + (ahead[b] >> 18);
      ok = false;
      for (int i = 0; i < waits && !ok; ++i) ok = wait(&q_empty[b], (n >> 1 & 1) ^ 1);
      if (!ok) break;
      const Work k = work_at(w);
      ahead[b] = stages_of(k);
      const int cols = cols_of(k);
      auto row_of = [&](int r) -> int64_t {
        int64_t row;
        int h;
        if constexpr (kCausal) {
          row = k.q_row0 + (k.row_base + r) / p.G;
          h = (k.row_base + r) % p.G;
        } else {
          row = (p.members ? p.members : inl.members)[k.member_base + r / p.G];
          h = r % p.G;
        }
        return ((int64_t)k.layer * p.n_rows_q + row) * p.Hq + k.kvh * p.G + h;
      };
      for (int i = lane; i < (kWide ? 2 : 1) * kKv4Rows; i += 32) {  // a group's rows from 0 or 64 on
        const int r = i < kKv4Rows ? i : i - kKv4Rows + cols;
        const bool has = i % kKv4Rows < cols && r < k.n_rows;
        meta.row[b][i] = has ? row_of(r) : -1;
        if constexpr (kCausal)
          meta.seen[b][i] = has ? k.L0 + (k.row_base + r) / p.G + 1 - k.page0 * kPageTokens : 0x7fffffff;
      }
      __syncwarp();
      uint8_t* to = base + b * C::kQBytes;
      auto place = [&](int i) -> uint4* {  // this lane's i-th 16 bytes
        const int x = (i * 32 + lane) / kChunks, c = lane % kChunks;
        const bool other = kWide && x >= cols;
        const int r = other ? x - cols : x;
        return reinterpret_cast<uint4*>(to + (other ? C::kQTile : 0) + (c >> 3) * kKv4Rows * 128 + r * 128 +
                                        (((c & 7) ^ (r & 7)) << 4));
      };
      auto own_at = [&](int i) {  // and its row's place in meta.own
        const int x = (i * 32 + lane) / kChunks;
        return kWide && x >= cols ? x - cols + kKv4Rows : x;
      };
      // All in flight at once, and in short loops, since a block's first queries are loaded
      // by code that it has not run (133 rows onto 23041: 115.6 -> 111.6 us; by eights through registers before).
      const int mine = (kWide ? 2 : 1) * cols * kChunks / 32;  // a multiple of 4
#pragma unroll 2
      for (int i = 0; i < mine; ++i) {
        const int x = (i * 32 + lane) / kChunks;
        const int64_t row = meta.row[b][kWide && x >= cols ? x - cols + kKv4Rows : x];
        copy16_async(place(i), p.q + (row >= 0 ? row * D + lane % kChunks * 8 : 0), row >= 0);
      }
      copies_wait();
      // The largest finite magnitude of 16 bytes, as bf16 bits.
      auto top_of = [](const uint4& v) -> uint32_t {
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
        uint32_t two = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t a = x[e] & 0x7fff7fffu;
          two = __vmaxu2(two, a & ~__vcmpgeu2(a, 0x7f807f80u));
        }
        return max(two & 0xffffu, two >> 16);
      };
      auto unlike_by = [](uint32_t most, uint32_t least) { return (int)(most >> 7) - (int)(least >> 7) > kAlike; };
      // Of all rows the most, and (zeros aside) the least: of any 16 bytes first, since no row's is below that.
      uint32_t most = 0, least = 0xffffffffu;
#pragma unroll 2
      for (int i = 0; i < mine; ++i) {
        const uint32_t top = top_of(*place(i));
        most = max(most, top);
        least = min(least, top - 1u);
      }
      most = __reduce_max_sync(0xffffffffu, most);
      bool unlike = most > 0 && unlike_by(most, __reduce_min_sync(0xffffffffu, least) + 1u);
      if (unlike) {  // each row's own
        least = 0xffffffffu;
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
          uint32_t top = top_of(*place(i));
#pragma unroll
          for (int h = 1; h < kChunks; h *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, h));
          least = min(least, top - 1u);
          if (lane % kChunks == 0) meta.own[b][own_at(i)] = __uint_as_float(top);
        }
        unlike = unlike_by(most, __reduce_min_sync(0xffffffffu, least) + 1u);
      }
      // by 2^e the largest comes to [2^13, 2^14)
      auto power = [](uint32_t top) { return min(100, 140 - (int)max(top >> 7, 1u)); };
      auto two_to = [](int e) { return __uint_as_float((uint32_t)(e + 127) << 23); };
      const int all = unlike ? 0 : power(most);
      if (lane == 0) {
        const float x = p.scale_log2 * 16.f * two_to(-all);
        meta.scale[b] = unlike ? -x : x;
      }
      __syncwarp();
#pragma unroll 2
      for (int i = 0; i < mine; ++i) {
        const uint4 v = *place(i);
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
        int e = all;
        if (unlike) {
          float* own = &meta.own[b][own_at(i)];
          e = power(__float_as_uint(*own));
          __syncwarp();
          if (lane % kChunks == 0) *own = -two_to(-e);
        }
        const float by = two_to(e);
        uint32_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          y[j] = as_u32(__floats2half2_rn(__uint_as_float(x[j] << 16) * by, __uint_as_float(x[j] & 0xffff0000u) * by));
        *place(i) = make_uint4(y[0], y[1], y[2], y[3]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[b]);
    }
    timeout(ok, lane);
  }

  // ---- softmax --------------------------------------------------------------------------
  // A group's stages of a work, for up to kCols rows (g0 stages before it in the
  // block), and half of its results.  False when a wait of any warp ran out.
  template <int kCols, bool kUnlike = false>
  __device__ __forceinline__ bool softmax(const Work& k, int n, int g0, int group, int warp, int lane) {
    const int key = warp * 32 + lane, qb = n & 1, stages = stages_of(k), id = 1 + group;
    const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
    const uint32_t s_at = mine + kTmemS + group * 64, o_at = mine + kTmemO + group * 64;
    float* ref = meta.m[group];
    float* factor = meta.f[group];
    auto& red = meta.red[group];
    const int r0 = kWide ? group * kKv4Rows : 0;
    const int32_t* seen = meta.seen[qb] + r0;
    // a narrow work ends at a barrier of both groups, where the other may wait already
    auto fails = [] {
      if constexpr (!kWide) any_of<256>(3, true);
      return false;
    };
    float l[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) l[i] = 0.f;
    bool ok = wait(&q_full[qb], n >> 1 & 1);  // the rows' places and the scale
    const float c = *reinterpret_cast<volatile float*>(&meta.scale[qb]);
    bool first = true;
    for (int t = kWide ? 0 : (g0 ^ group) & 1; t < stages; t += kStep) {
      const uint32_t x = turn(g0 + t);
      ok = ok && wait(&s_full[group], x);
      tc_fence_after_sync();
      const int at = t * kKv4Keys + key;  // this thread's key in the run
      bool masks;
      if constexpr (kCausal) masks = (t + 1) * kKv4Keys > seen[0];  // the first row sees the fewest
      else masks = (t + 1) * kKv4Keys > k.n_keys;
      if constexpr (kUnlike) {  // each row's scores by its own share of the scale, where they lie
        const float* own = meta.own[qb] + r0;
#pragma unroll 1
        for (int j = 0; j < kCols; j += 8) {
          float y[8];
          tmem_ld8(s_at + j, y);
          uint32_t u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(y[i] * own[j + i]);
          tmem_st8u_nowait(s_at + j, u);
        }
        tmem_wait_st();
      }
      float s[kCols];  // over the rows' references, keys that a row does not see hidden
      // A second time where a reference has moved (the scores are computed in one place,
      // since another would need as many registers again), and no third.
      bool moved = false;
#pragma unroll 1
      for (;;) {
        tmem_ld_cols<kCols>(s_at, s);
#pragma unroll
        for (int i = 0; i < kCols; i += 4) {
          const float4 m = *reinterpret_cast<const float4*>(&ref[i]);
          const float2 y = __ffma2_rn(make_float2(s[i], s[i + 1]), make_float2(c, c), make_float2(m.x, m.y));
          const float2 z = __ffma2_rn(make_float2(s[i + 2], s[i + 3]), make_float2(c, c), make_float2(m.z, m.w));
          s[i] = y.x, s[i + 1] = y.y, s[i + 2] = z.x, s[i + 3] = z.y;
        }
        if (masks) {
#pragma unroll
          for (int i = 0; i < kCols; ++i)
            if (kCausal ? at >= seen[i] : at >= k.n_keys) s[i] = -INFINITY;
        }
        float a = s[0], b = s[1];
#pragma unroll
        for (int i = 2; i + 3 < kCols; i += 4) a = fmax3(a, s[i], s[i + 1]), b = fmax3(b, s[i + 2], s[i + 3]);
        const float highest = fmax3(a, b, fmaxf(s[kCols - 2], s[kCols - 1]));
        if (!any_of<128>(id, first || !ok || highest > kHeadroom)) break;
        if (any_of<128>(id, !ok)) return fails();
        if (moved) {  // scores of 10^7 and more, which fp32 has off by as much: these keys alike
#pragma unroll
          for (int i = 0; i < kCols; ++i) s[i] = s[i] > kHeadroom ? kHeadroom : s[i];
          break;
        }
#pragma unroll 1
        for (int j = 0; j < kCols; j += 8) {
          float y[8];
          tmem_ld8(s_at + j, y);
#pragma unroll
          for (int i = 0; i < 8; ++i) {  // in an order of whole numbers, which the warp reduces at once
            float v = y[i] * c;
            if (masks && (kCausal ? at >= seen[j + i] : at >= k.n_keys)) v = -INFINITY;
            const int o = __float_as_int(v);
            const int top = __reduce_max_sync(0xffffffffu, o ^ (o >> 31 & 0x7fffffff));
            if (lane == i) red[warp][j + i] = top;
          }
        }
        named_barrier_sync(id, 128);
        if (key < kCols) {
          int o = max(max(red[0][key], red[1][key]), max(red[2][key], red[3][key]));
          o ^= o >> 31 & 0x7fffffff;
          const float top = __int_as_float(o), old = first ? kUnset : -ref[key];
          // Below the maximum by what fp32 may have it off as well, and never lower than it was
          // (a NaN stays one).
          const float to = top - kBelow - fabsf(top) * kOff;
          const bool moves = first ? top != -INFINITY : top - old > kHeadroom && !(to < old);
          const float m = moves ? to : old;
          ref[key] = -m;
          factor[key] = moves ? ex2(old - m) : 1.f;
        }
        // O as the stages before left it
        if (!first) ok = wait(&pv_done[group], x ^ 1);
        if (any_of<128>(id, !ok)) return fails();
        if (!first) {
          tc_fence_after_sync();
#pragma unroll
          for (int i = 0; i < kCols; ++i) l[i] *= factor[i];
#pragma unroll 1
          for (int j = 0; j < kCols; j += 8) {
            float o[8];
            tmem_ld8(o_at + j, o);
            uint32_t u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(o[i] * factor[j + i]);
            tmem_st8u_nowait(o_at + j, u);
          }
          tmem_wait_st();
        }
        first = false;
        moved = true;
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_empty[group]);
      ok = ok && wait(&pv_done[group], x ^ 1);  // the group's P before has been read
      uint8_t* to = base + C::kOffP + group * C::kPBytes + key * 128;
#pragma unroll
      for (int j = 0; j < kCols / 8; ++j) {
        const float* v = s + 8 * j;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float2 e = make_float2(ex2(v[i]), ex2(v[i + 1]));
          const float2 sum = __fadd2_rn(make_float2(l[8 * j + i], l[8 * j + i + 1]), e);
          l[8 * j + i] = sum.x, l[8 * j + i + 1] = sum.y;
          w[i / 2] = as_u32(__floats2half2_rn(e.x, e.y));
        }
        *reinterpret_cast<uint4*>(to + ((j ^ (key & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      fence_proxy_async_smem();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[group]);
    }
    // ---- the work's results: sums over the keys, O of both groups out of tensor memory
    if (any_of<128>(id, !ok)) return fails();
    if (first) {  // the group has had none of its stages
      if (key < kCols) meta.sum[group][key] = 0.f;
    } else {
#pragma unroll
      for (int j = 0; j < kCols; j += 16) {
        constexpr int kLast = kCols % 16 ? kCols - 8 : kCols;
        const int some = j == kLast ? 8 : 16;
        float* a = l + j;  // after these steps lane i has column i % some
#pragma unroll
        for (int h = some / 2; h; h >>= 1)
#pragma unroll
          for (int i = 0; i < h; ++i) {
            const bool up = lane & h;
            const float give = up ? a[i] : a[i + h], keep = up ? a[i + h] : a[i];
            a[i] = keep + __shfl_xor_sync(0xffffffffu, give, h);
          }
        for (int h = some; h < 32; h *= 2) a[0] += __shfl_xor_sync(0xffffffffu, a[0], h);
        if (lane < some) red[warp][j + lane] = __float_as_int(a[0]);
      }
      named_barrier_sync(id, 128);
      if (key < kCols)
        meta.sum[group][key] = (__int_as_float(red[0][key]) + __int_as_float(red[1][key])) +
                                (__int_as_float(red[2][key]) + __int_as_float(red[3][key]));
    }
    const int64_t stride = kCausal && k.split < 0 ? D : (int64_t)p.max_splits * D;
    float* part = p.part_o + (int64_t)k.split * D + key;
    const int64_t* rows = meta.row[qb] + r0;
    auto put_lse = [&](int i, float m, float sum) {  // 0: the row sees none of these keys
      const int64_t row = rows[i];
      if (row < 0) return;
      const float lse = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
      if (kCausal && k.split < 0) p.lse[row] = lse;
      else p.part_lse[row * p.max_splits + k.split] = lse;
    };
    auto put_o = [&](int64_t row, float y) {
      if (kCausal && k.split < 0) p.o[row * stride + key] = __float2bfloat16_rn(y);
      else part[row * stride] = y;
    };
    const int g1 = g0 + stages - 1;
    if constexpr (kWide) {
      ok = wait(&pv_done[group], turn(g1));
      if (any_of<128>(id, !ok)) return fails();
      tc_fence_after_sync();
      if (key < kCols) {
        const float sum = meta.sum[group][key];
        factor[key] = sum == 0.f ? 0.f : 16.f / sum;
        put_lse(key, -ref[key], sum);
      }
      named_barrier_sync(id, 128);
#pragma unroll 1
      for (int j = 0; j < kCols / 8; ++j) {
        float a[8];
        tmem_ld8(o_at + 8 * j, a);
        if (key < D) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int64_t row = rows[8 * j + i];
            if (row < 0) break;  // rows are in order: none beyond
            const float f = factor[8 * j + i];
            put_o(row, f == 0.f ? 0.f : a[i] * f);
          }
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&o_empty[group]);
        mbar_arrive(&q_empty[qb]);
      }
      named_barrier_sync(id, 128);  // all have read factors and references before the next work writes them
      return true;
    }
    // both streams' last P V (the last stage's, and that of the stage before it, the other stream's)
    ok = wait(&pv_done[g1 & 1], g1 >> 1 & 1) && (stages == 1 || wait(&pv_done[~g1 & 1], (g1 - 1) >> 1 & 1));
    if (any_of<256>(3, !ok)) return false;
    tc_fence_after_sync();
    // this group's half of the rows (by eights), with factors for O of both streams
    constexpr int kHalf = (kCols + 15) / 16 * 8;
    const int c0 = group * kHalf, mine_n = group ? kCols - kHalf : kHalf;
    if (key < mine_n) {
      const int i = c0 + key;
      const float ma = meta.sum[0][i] == 0.f ? -INFINITY : -meta.m[0][i];
      const float mb = meta.sum[1][i] == 0.f ? -INFINITY : -meta.m[1][i], m = fmaxf(ma, mb);
      const float fa = meta.sum[0][i] == 0.f ? 0.f : ex2(ma - m), fb = meta.sum[1][i] == 0.f ? 0.f : ex2(mb - m);
      const float sum = fa * meta.sum[0][i] + fb * meta.sum[1][i];
      const float over = sum == 0.f ? 0.f : 16.f / sum;
      meta.f[0][i] = fa * over;
      meta.f[1][i] = fb * over;
      put_lse(i, m, sum);
    }
    named_barrier_sync(id, 128);
#pragma unroll 1
    for (int c1 = c0; c1 < c0 + mine_n; c1 += 8) {
      float a[8], b[8];
      tmem_ld8(mine + kTmemO + c1, a);
      tmem_ld8(mine + kTmemO + 64 + c1, b);
      if (key < D) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int64_t row = rows[c1 + i];
          if (row < 0) break;  // rows are in order: none beyond
          const float fa = meta.f[0][c1 + i], fb = meta.f[1][c1 + i];
          // O of a group that has had no stage is what a work before left there
          put_o(row, (fa == 0.f ? 0.f : a[i] * fa) + (fb == 0.f ? 0.f : b[i] * fb));
        }
      }
    }
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(o_empty);
      mbar_arrive(&q_empty[qb]);
    }
    named_barrier_sync(3, 256);  // all have read factors and references before the next work writes them
    return true;
  }

  __device__ __forceinline__ void softmax_all(int stream, int warp, int lane) {
    int g = 0, n = 0;
    bool ok = true;
    for (int w = blockIdx.x; ok && w < n_works; w = after(w, n++)) {
      const Work k = work_at(w);
      // eights of rows: what the products have beyond them counts for nothing
      const int rows = kWide ? min(cols_of(k), k.n_rows - stream * cols_of(k)) : k.n_rows;
      // unlike rows, of any number, in a copy that scales each by itself
      const bool there = wait(&q_full[n & 1], n >> 1 & 1);
      timeout(there, lane);
      if (there && *reinterpret_cast<volatile float*>(&meta.scale[n & 1]) < 0.f)
        ok = softmax<64, true>(k, n, g, stream, warp, lane);
      else if (rows <= 16) ok = softmax<16>(k, n, g, stream, warp, lane);
      else if (rows <= 24) ok = softmax<24>(k, n, g, stream, warp, lane);
      else if (rows <= 32) ok = softmax<32>(k, n, g, stream, warp, lane);
      else if (rows <= 40) ok = softmax<40>(k, n, g, stream, warp, lane);
      else if (rows <= 48) ok = softmax<48>(k, n, g, stream, warp, lane);
      else ok = softmax<64>(k, n, g, stream, warp, lane);
      g += stages_of(k);
    }
    timeout(ok, lane);
  }
};

template <int D, bool kCausal, bool kWide>
__global__ void __launch_bounds__(kThreads, 1)
    kv4_attend_kernel(const __grid_constant__ Kv4AttnParams p, const __grid_constant__ InlineDecodePlan inl) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* base = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Kernel<D, kCausal, kWide> k(p, inl, base);
  if (warp == kMmaWarp) tmem_alloc(&k.meta.tmem, kTmemCols);
  if (threadIdx.x == 0) k.init_barriers();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  k.tmem = k.meta.tmem;
  griddep_wait();
  griddep_launch_dependents();
  // Each role ends in a branch of its own: behind a common end the compiler could
  // use registers that a role has given back.
  auto done = [&] {
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
  };
  using R = Regs<kCausal, kWide>;
  if (warp < kUnpackWarp) {
    set_registers<R::kSoft>();
    k.softmax_all(warp >> 2, warp & 3, lane);
    done();
  } else if (warp < kLoadWarp) {
    set_registers<R::kUnpack>();
    k.unpack((warp - kUnpackWarp) >> 2, warp & 3, lane);
    done();
  } else {
    set_registers<R::kAux>();
    if (warp == kLoadWarp) k.load(lane);
    else if (warp == kQWarp) k.queries(lane);
    else k.issue(warp - kMmaWarp, lane);
    done();
    if (warp == kMmaWarp) {
      tc_fence_after_sync();
      tmem_dealloc(k.tmem, kTmemCols);
    }
  }
}

template <int D, bool kCausal, bool kWide>
cudaError_t launch_t(const Kv4AttnParams& p, const InlineDecodePlan& inl, cudaStream_t s) {
  static std::mutex mu;
  static int sms_of[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::unique_lock<std::mutex> lock(mu);
  if (!sms_of[dev]) {
    e = cudaFuncSetAttribute(kv4_attend_kernel<D, kCausal, kWide>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             Cfg<D, kWide>::kSmemBytes);
    if (e != cudaSuccess) return e;
    int n = 0;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, kv4_attend_kernel<D, kCausal, kWide>);
    if (e != cudaSuccess) return e;
    if (!Regs<kCausal, kWide>::suffice(fa.numRegs)) return cudaErrorInvalidKernelImage;
    sms_of[dev] = n;
  }
  const int sms = sms_of[dev];
  lock.unlock();
  const int64_t works = (int64_t)p.n_items * p.Hkv * p.L;
  if (works > (1 << 30)) return cudaErrorInvalidValue;
  const int grid = (int)(works < sms ? works : sms);
  return launch_chained(kv4_attend_kernel<D, kCausal, kWide>, dim3(grid), dim3(kThreads), Cfg<D, kWide>::kSmemBytes, s, p, inl);
}

template <int D>
cudaError_t launch_d(const Kv4AttnParams& p, const InlineDecodePlan& inl, cudaStream_t s) {
  if (p.tiles) return p.wide ? launch_t<D, true, true>(p, inl, s) : launch_t<D, true, false>(p, inl, s);
  return p.wide ? launch_t<D, false, true>(p, inl, s) : launch_t<D, false, false>(p, inl, s);
}

}  // namespace

cudaError_t launch_kv4_attend(const Kv4AttnParams& p, const InlineDecodePlan* inl, int D, cudaStream_t s) {
  static const InlineDecodePlan kNone{};
  const InlineDecodePlan& ip = inl ? *inl : kNone;
  if (p.n_items <= 0) return cudaSuccess;
  if (D == 128) return launch_d<128>(p, ip, s);
  if (D == 64) return launch_d<64>(p, ip, s);
  return cudaErrorInvalidValue;
}

}  // namespace st
