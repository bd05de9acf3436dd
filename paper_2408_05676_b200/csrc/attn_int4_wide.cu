// Attention of a step's rows over a 4-bit paged cache (int4.cuh) with heads of 128, on tcgen05 and tensor memory:
// o = sum_t p_t v_t / sum_t p_t, p_t = exp(q . k_t / sqrt(dh)); row i sees the cached tokens and, of the step's own rows, 0 .. i (chain) or
// its ancestors and itself (token tree).
//
// The rows of a sequence that share a kv head (rows x n_heads / n_kv_heads) form tiles of up to 48.  (sequence, kv head, row tile) is a
// unit; its tokens come in blocks of 128, and all units' blocks, one after another, are divided evenly over the SMs, a CTA each, so that
// ragged lengths leave nobody idle.  Tokens are the 128 lanes of S^T = K Q^T and features those of O^T += V^T P^T, so that few rows
// waste little of an MMA.  Codes go from shared memory through registers straight into tensor memory as the A operands: unpacked keys
// and values never cross shared memory, whose bandwidth (128 bytes a clock; 64 KB a block to write, as many to read) would be the bound.
//   warps 0-3   keys: a thread a token; 64 columns of bf16 pairs
//   warps 4-7   values: a thread a feature; pairs of tokens
//   warps 8-11  softmax: a thread a token; P^T to shared memory (the B operand); a unit's end
//   warp 12     copies: a page's K and V of a head, codes and scales, are one bulk copy; Q
//   warp 13     MMAs.  The sums of P are a product with ones, in accumulators of their own.
// What bounds it: each scheduler has one warp of each kind, and the three unpacking and softmax warps issue 600 .. 900 instructions a
// block; a block's 20 KB take 860 clocks of an SM's share of HBM.
//
// The softmax's reference m is a whole number in the exponent of two: raising it multiplies p and O by powers of two, exactly, so a
// row's result does not depend on where its walk was cut but for the order of fp32 sums.  It is raised only when a score exceeds it by
// more than 2^6; p stays below 2^7.
//
// A CTA leaves pieces (m, sum, O in fp32) of the units at its two ends if those go on in other CTAs; whichever of a unit's CTAs arrives last
// joins them in the order of the tokens.  Nothing waits for another CTA.
// Tensor memory is allocated after everything before this kernel has ended, and the CTA's shared memory leaves no room for another
// kernel's CTA that allocates any, so that no two wait for each other's columns.
#include <algorithm>

#include "attn_int4.cuh"
#include "umma.cuh"

namespace laser {
namespace {

using bf16 = __nv_bfloat16;
constexpr int kDh = 128, kBlk = q4_block_bytes(kDh);
constexpr int kPages = 8;              // of a block: 128 tokens
constexpr int kStages = 6;             // blocks of codes in shared memory
constexpr int kStage = kPages * kBlk;
constexpr int kThreads = 14 * 32;
constexpr int kMostRows = 48;

template <int NP>
struct Wide {
  static constexpr int kUnits = NP <= 32 ? 2 : 1;       // accumulators of units at a time
  static constexpr int kRowsBytes = NP * kDh * 2;       // Q, or P^T of a block: two swizzled halves of NP rows of 128 bytes
  static constexpr int kRecord = NP * kDh + 2 * NP;     // floats of a piece: O [row][feature], then (m, sum) of the rows
  // tensor memory columns
  static constexpr int kK = 0, kV = 128, kS = 256, kO = kS + 2 * NP, kL = kO + kUnits * NP, kOnes = 504;
  static_assert(kL + kUnits * NP <= kOnes, "tensor memory");
  static int smem(int B) { return 1024 + kStages * kStage + 4 * kRowsBytes + (B + 1) * 8 + B * 12; }
};

// where a block is: its sequence, kv head, row tile, and number in the unit; the sequence's row tiles, blocks of a unit and pages
struct Walk {
  int b, hk, rt, blk, tiles, blocks, pages;
};
struct Open { int b, hk, row0, start, blocks; };     // a unit that other CTAs have pieces of; its first block, from this CTA's first

__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                 "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t at, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// A in tensor memory, B in shared memory.  Four K steps in one piece of code: of operands that each MMA gets from ordinary registers every one
// is first moved to a uniform one, 90 clocks an MMA in all.
__device__ __forceinline__ void umma_ts4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t elected) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 b1, b2, b3;\n.reg .b32 a1, a2, a3;\nsetp.ne.b32 q, %5, 0;\nsetp.ne.b32 p, %4, 0;\n"
      "add.s64 b1, %2, 2;\nadd.s64 b2, %2, 4;\nadd.s64 b3, %2, 6;\nadd.s32 a1, %1, 8;\nadd.s32 a2, %1, 16;\nadd.s32 a3, %1, 24;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, 1;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, 1;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, 1;\n}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
// `steps` (1 .. 4) K steps of two products with one B: of a, 8 columns a step, into d, and of ones, always the same columns, into l
__device__ __forceinline__ void umma_ts_sums(uint32_t d, uint32_t l, uint32_t a, uint32_t ones, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t steps,
                                             uint32_t elected) {
  asm volatile(
      "{\n.reg .pred p, q, q1, q2, q3;\n.reg .b64 b1, b2, b3;\n.reg .b32 a1, a2, a3;\nsetp.ne.b32 q, %8, 0;\nsetp.ne.b32 p, %6, 0;\n"
      "setp.gt.and.u32 q1, %7, 1, q;\nsetp.gt.and.u32 q2, %7, 2, q;\nsetp.gt.and.u32 q3, %7, 3, q;\n"
      "add.s64 b1, %4, 2;\nadd.s64 b2, %4, 4;\nadd.s64 b3, %4, 6;\nadd.s32 a1, %2, 8;\nadd.s32 a2, %2, 16;\nadd.s32 a3, %2, 24;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], %4, %5, p;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%1], [%3], %4, %5, p;\n"
      "@q1 tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %5, 1;\n"
      "@q1 tcgen05.mma.cta_group::1.kind::f16 [%1], [%3], b1, %5, 1;\n"
      "@q2 tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %5, 1;\n"
      "@q2 tcgen05.mma.cta_group::1.kind::f16 [%1], [%3], b2, %5, 1;\n"
      "@q3 tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %5, 1;\n"
      "@q3 tcgen05.mma.cta_group::1.kind::f16 [%1], [%3], b3, %5, 1;\n}"
      ::"r"(d), "r"(l), "r"(a), "r"(ones), "l"(b), "r"(idesc), "r"(accumulate), "r"(steps), "r"(elected) : "memory");
}
// A bounded wait of a whole warp, in little code: five kinds of warps share the instruction caches, and loops that do not fit them run at a
// third of their speed.  A try that fails has suspended the warp for about a microsecond.
__device__ __forceinline__ bool await(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  int tries = 0;
  while (!__all_sync(0xffffffffu, mbar_try(bar, parity))) {
    if (++tries > (1 << 21)) *abort_flag = 1;
    if (*abort_flag) return false;
  }
  return true;
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// of the softmax warps: whether any thread says so
__device__ __forceinline__ bool group_any(bool x) {
  uint32_t y;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbar.red.or.pred q, 1, 128, p;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(y) : "r"(uint32_t(x)) : "memory");
  return y != 0;
}
__device__ __forceinline__ void group_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int NP>
__global__ void __launch_bounds__(kThreads, 1)
attn_int4_wide_kernel(const AttnArgs a) {
  using Z = Wide<NP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* const s_q = smem + kStages * kStage;                     // [2] Q: rows of 128 bytes, 64 features a half  (kStage is a multiple of 1024)
  uint8_t* const s_p = s_q + 2 * Z::kRowsBytes;                     // [2] P^T: 64 tokens a half
  long long* const s_pre = reinterpret_cast<long long*>(s_p + 2 * Z::kRowsBytes);   // [B + 1] blocks before a sequence
  int* const s_ctx = reinterpret_cast<int*>(s_pre + a.B + 1);       // [B]
  int* const s_nr = s_ctx + a.B;                                    // [B]
  int* const s_seq = s_nr + a.B;                                    // [B]
  __shared__ uint64_t raw_full[kStages], raw_empty[kStages], q_full[2], q_free[2], k_full[2], v_full[2], s_full[2], s_free[2], p_full[2], pv_done[2], o_free[2];
  // rows of units, three at a time: a warp may have begun the next but one while another still ends the first
  __shared__ long long s_sum[kThreads / 32], s_off[3][NP];          // (s_off:) a row's place in out
  __shared__ unsigned long long s_path[2][64];                      // a token tree's: the rows that a row sees
  __shared__ __align__(16) float s_shift[3][NP];
  __shared__ float s_down[NP], s_top[4][NP];                        // (s_shift:) -m; what O is multiplied with; a block's largest scores by warp
  __shared__ int s_row[3][NP];                                      // the step's row that a row is of
  __shared__ Open s_open[2];
  __shared__ int s_abort, s_last[2];
  __shared__ uint32_t s_tmem;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  next_may_launch();
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&raw_full[i]), 1); mbar_init(smem_u32(&raw_empty[i]), 8); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&q_full[i]), 1); mbar_init(smem_u32(&q_free[i]), 1);
      mbar_init(smem_u32(&k_full[i]), 4); mbar_init(smem_u32(&v_full[i]), 4);
      mbar_init(smem_u32(&s_full[i]), 1); mbar_init(smem_u32(&s_free[i]), 4);
      mbar_init(smem_u32(&p_full[i]), 4); mbar_init(smem_u32(&pv_done[i]), 1); mbar_init(smem_u32(&o_free[i]), 4);
      s_open[i].b = -1;
    }
    mbar_fence_init();
  }
  // a step's tables were complete before any kernel of the forward began
  if (!a.row_ctx) wait_for_earlier();

  // ---- the units: blocks of all sequences, one after another ----
  auto tiles_of = [&](int nr) { return (nr * a.G + NP - 1) / NP; };
  auto pages_of = [&](int b) { return (s_ctx[b] + s_nr[b] + 15) >> 4; };
  long long total = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + tid;
    int ctx = 0, nr = 0, seq = 0;
    if (b < a.B) {
      seq = a.seq_ids[b];
      if (a.row_ctx) {
        ctx = a.row_ctx[b]; nr = a.row_n[b];
      } else {
        nr = min(max(a.n_rows[b], 0), a.Rs);
        if (seq < 0 || seq >= a.max_seqs) {
          if (nr > 0 && blockIdx.x == 0) atomicCAS(a.status, 0, LASER_ERR_INVALID_ARG);
          nr = 0;
        } else {
          ctx = a.seq_len[seq];
          if (nr > 0 && (ctx < 0 || nr > a.capacity - ctx)) {
            if (blockIdx.x == 0) atomicCAS(a.status, 0, LASER_ERR_CAPACITY);
            nr = 0;
          }
        }
      }
      s_ctx[b] = ctx; s_nr[b] = nr; s_seq[b] = seq;
    }
    const long long mine = nr > 0 ? (long long)(a.Hkv * tiles_of(nr)) * ((ctx + nr + 127) >> 7) : 0;
    long long x = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) s_sum[warp] = x;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w == warp) x += all;
      all += s_sum[w];
    }
    if (b < a.B) s_pre[b] = total + x - mine;
    total += all;
    __syncthreads();
  }
  if (a.row_ctx) wait_for_earlier();
  const int per_cta = total <= 0xffffffffll ? int((unsigned(total) + gridDim.x - 1) / gridDim.x) : int((total + gridDim.x - 1) / gridDim.x);
  const long long c0 = (long long)per_cta * blockIdx.x;
  if (c0 >= total) return;
  const int n = int(min(total - c0, (long long)per_cta));            // this CTA's blocks
  float* const my_part = a.part + size_t(2 * blockIdx.x) * Z::kRecord;

  if (warp == 13) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  const uint32_t lanes = tmem + (uint32_t((warp & 3) * 32) << 16);    // this warp's lanes
  if (warp < 4) {
    const uint32_t ones[8] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
    tmem_st8(lanes + Z::kOnes, ones);       // (the MMAs wait for these warps' first block)
  }

  Walk w;
  {
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_pre[mid] <= c0) lo = mid; else hi = mid - 1;
    }
    w.b = lo; w.pages = pages_of(lo); w.tiles = tiles_of(s_nr[lo]); w.blocks = (w.pages + kPages - 1) / kPages;
    const unsigned at = unsigned(c0 - s_pre[lo]), unit = at / unsigned(w.blocks);
    w.blk = int(at - unit * w.blocks);
    w.hk = int(unit / unsigned(w.tiles));
    w.rt = int(unit - w.hk * w.tiles);
  }
  auto next = [&](Walk& x) {        // to the next block; whether that begins a unit
    if (++x.blk < x.blocks) return false;
    x.blk = 0;
    if (++x.rt == x.tiles) {
      x.rt = 0;
      if (++x.hk == a.Hkv) {
        x.hk = 0;
        do { ++x.b; } while (x.b < a.B && s_nr[x.b] == 0);
        if (x.b < a.B) { x.pages = pages_of(x.b); x.tiles = tiles_of(s_nr[x.b]); x.blocks = (x.pages + kPages - 1) / kPages; }
      }
    }
    return true;
  };
  auto verify_row = [&](int row) { return a.G == 1 ? row : int(__umulhi(unsigned(row), a.group_inv)); };
  bool ok = true;

  if (warp < 4) {
    // ---- keys ----
    const int page = tid >> 4, t = tid & 15;
#pragma unroll 1
    for (int i = 0, st = 0, round = 0; i < n; ++i) {
      const int bf = i & 1, np = min(kPages, w.pages - w.blk * kPages);
      ok = await(smem_u32(&raw_full[st]), round, &s_abort);
      if (ok && i >= 2) ok = await(smem_u32(&s_full[bf]), ((i >> 1) - 1) & 1, &s_abort);      // (the MMA that read this buffer)
      if (!ok) break;
      fence_after();
      if (2 * warp < np) {          // (of a warp's two pages one may be missing: what its tokens get is masked)
        const uint8_t* raw = smem + st * kStage + page * kBlk;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          const uint32_t sz = *reinterpret_cast<const uint32_t*>(raw + q4_k_scale(kDh, t, 0) + 4 * c);
          const uint4 k = *reinterpret_cast<const uint4*>(raw + q4_k_codes(kDh, t, 0) + 256 * c);
          const uint32_t s2 = __byte_perm(sz, 0, 0x1010), z2 = __byte_perm(sz, 0, 0x3232);
          const uint32_t ks[4] = {k.x, k.y, k.z, k.w};
          uint32_t v[16];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            v[4 * x] = values(ks[x], s2, z2);
            v[4 * x + 1] = values(__funnelshift_r(ks[x], ks[x], 4), s2, z2);
            v[4 * x + 2] = values(__funnelshift_r(ks[x], ks[x], 8), s2, z2);
            v[4 * x + 3] = values(__funnelshift_r(ks[x], ks[x], 12), s2, z2);
          }
          tmem_st16(lanes + Z::kK + bf * 64 + c * 16, v);
        }
      }
      tmem_st_wait();
      fence_before();
      __syncwarp();
      if (lane == 0) { mbar_arrive(smem_u32(&raw_empty[st])); mbar_arrive(smem_u32(&k_full[bf])); }
      if (++st == kStages) { st = 0; round ^= 1; }
      next(w);
    }
  } else if (warp < 8) {
    // ---- values ----
    const int c = tid - 128, turn = (4 * (c & 3) + 29) & 31;       // its nibble to bits 3 .. 6
#pragma unroll 1
    for (int i = 0, st = 0, round = 0; i < n; ++i) {
      const int bf = i & 1, np = min(kPages, w.pages - w.blk * kPages);
      ok = await(smem_u32(&raw_full[st]), round, &s_abort);
      if (ok && i >= 2) ok = await(smem_u32(&pv_done[bf]), ((i >> 1) - 1) & 1, &s_abort);
      if (!ok) break;
      fence_after();
      const uint8_t* raw = smem + st * kStage;
#pragma unroll 1
      for (int p = 0; p < np; ++p, raw += kBlk) {
        const uint4 c0_ = *reinterpret_cast<const uint4*>(raw + q4_v_codes(kDh, 0, c >> 2)), c1_ = *reinterpret_cast<const uint4*>(raw + q4_v_codes(kDh, 8, c >> 2));
        const uint32_t cs[8] = {c0_.x, c0_.y, c0_.z, c0_.w, c1_.x, c1_.y, c1_.z, c1_.w};
        uint32_t v[8];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint4 sz = *reinterpret_cast<const uint4*>(raw + q4_v_scale(kDh, 4 * x, warp & 3));      // s, z of two pairs of tokens
          v[2 * x] = values(__funnelshift_r(cs[2 * x], cs[2 * x], turn), sz.x, sz.y);
          v[2 * x + 1] = values(__funnelshift_r(cs[2 * x + 1], cs[2 * x + 1], turn), sz.z, sz.w);
        }
        tmem_st8(lanes + Z::kV + bf * 64 + p * 8, v);
      }
      tmem_st_wait();
      fence_before();
      __syncwarp();
      if (lane == 0) { mbar_arrive(smem_u32(&raw_empty[st])); mbar_arrive(smem_u32(&v_full[bf])); }
      if (++st == kStages) { st = 0; round ^= 1; }
      next(w);
    }
  } else if (warp < 12) {
    // ---- softmax ----
    const int tok = tid - 256;                     // token of a block, feature of a result
    const uint32_t p_at = uint32_t(tok >> 6) * (NP * 128) + (tok & 7) * 2, p_chunk = (tok & 63) >> 3;
    bool begins = true;
    int unit = 0, tb = 0, first = w.blk, path_b = -1, path_buf = 0;
    // a unit's result, or this CTA's piece of it
    auto finish = [&](const Walk& x, int i, int u, int tb, int from) {
      const int o_buf = Z::kUnits == 2 ? u & 1 : 0, na = min(NP, s_nr[x.b] * a.G - x.rt * NP);
      ok = await(smem_u32(&pv_done[i & 1]), (i >> 1) & 1, &s_abort) && ok;
      fence_after();
      const bool whole = from == 0 && x.blk + 1 == x.blocks;
      float* rec = my_part + (from == 0 ? 1 : 0) * Z::kRecord;
#pragma unroll
      for (int n0 = 0; n0 < NP; n0 += 16) {
        if (n0 >= na) break;
        uint32_t o[16], l[16];
        tmem_ld16(lanes + Z::kO + o_buf * NP + n0, o);
        tmem_ld16(lanes + Z::kL + o_buf * NP + n0, l);
        tmem_ld_wait();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (n0 + r >= na) break;
          const float ov = __uint_as_float(o[r]), lv = __uint_as_float(l[r]);
          if (whole) {
            a.out[s_off[tb][n0 + r] + tok] = __float2bfloat16(ov / lv);      // (a row sees itself: its sum is not zero)
          } else {
            __stcg(rec + (n0 + r) * kDh + tok, ov);
            if (tok == 0) {
              const float sh = s_shift[tb][n0 + r];
              __stcg(reinterpret_cast<float2*>(rec + NP * kDh) + n0 + r, make_float2(sh == kNothing ? -INFINITY : -sh, lv));
            }
          }
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&o_free[o_buf]));
      if (!whole && tok == 0) s_open[from == 0 ? 1 : 0] = Open{x.b, x.hk, x.rt * NP, i - x.blk, x.blocks};
    };
    Walk ended{};                                   // a unit whose end is put off until the next block is on its way
    int ended_i = -1, ended_first = 0;
    for (int i = 0; i < n; ++i) {
      const int bf = i & 1, row0 = w.rt * NP, ctx = s_ctx[w.b], nr = s_nr[w.b], na = min(NP, nr * a.G - row0);
      if (begins) {
        if (a.parents && path_b != w.b) {
          path_buf ^= 1;
          if (warp == 8) {
            unsigned long long path[2];
            tree_paths(a.parents + size_t(w.b) * a.Rs, nr, lane, path);
            s_path[path_buf][lane] = path[0];
            s_path[path_buf][lane + 32] = path[1];
          }
          path_b = w.b;
        }
        if (tok < NP) {
          const int row = row0 + tok, r = verify_row(row);
          s_row[tb][tok] = r;
          s_off[tb][tok] = (long long)(size_t(w.b) * a.Rs + r) * a.ldo + (w.hk * a.G + row - r * a.G) * kDh;
          s_shift[tb][tok] = tok < na ? kNothing : -kNothing;      // (rows that are not never raise anything)
        }
        group_sync();
      }
      ok = await(smem_u32(&s_full[bf]), (i >> 1) & 1, &s_abort) && ok;
      fence_after();
      // eight rows' scores of the thread's token
      const int rel = w.blk * 128 + tok - ctx;      // from 0 on: one of the step's own rows, or a slot behind them
      const bool masked = w.blk * 128 + 127 >= ctx;
      auto scores = [&](int r0, float (&x)[8]) {
        uint32_t v[8];
        tmem_ld8(lanes + Z::kS + bf * NP + r0, v);
        tmem_ld_wait();
#pragma unroll
        for (int r = 0; r < 8; ++r) x[r] = __uint_as_float(v[r]);
        if (masked && rel >= 0) {
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int row = r0 + r < na ? s_row[tb][r0 + r] : 0;
            const bool on = a.parents ? rel < 64 && (s_path[path_buf][row] >> (rel & 63) & 1) : rel <= row;
            if (!on) x[r] = -INFINITY;
          }
        }
      };
      bool above = begins || !ok;
#pragma unroll 1
      for (int r0 = 0; r0 < na; r0 += 8) {
        float x[8];
        scores(r0, x);
        const float4 h0 = *reinterpret_cast<const float4*>(&s_shift[tb][r0]), h1 = *reinterpret_cast<const float4*>(&s_shift[tb][r0 + 4]);
        const float hs[8] = {h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w};
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 8; ++r) top = fmaxf(top, fmaf(x[r], a.scale, hs[r]));
        above = above || top > 6.f;
      }
      if (group_any(above)) {
        if (group_any(!ok)) { ok = false; break; }
#pragma unroll 1
        for (int r0 = 0; r0 < na; r0 += 8) {
          float x[8];
          scores(r0, x);
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float top = warp_max(x[r]);
            if (lane == 0) s_top[warp & 3][r0 + r] = top;
          }
        }
        group_sync();
        if (tok < na) {
          const float top = fmaxf(fmaxf(s_top[0][tok], s_top[1][tok]), fmaxf(s_top[2][tok], s_top[3][tok]));
          const float old = s_shift[tb][tok], now = fminf(old, -ceilf(top * a.scale));
          s_shift[tb][tok] = now;
          s_down[tok] = ex2(now - old);
        }
        group_sync();
        if (!begins) {                              // O and the sums so far, when the MMAs before have ended
          ok = await(smem_u32(&pv_done[bf ^ 1]), ((i - 1) >> 1) & 1, &s_abort) && ok;
          fence_after();
          const int o_buf = Z::kUnits == 2 ? unit & 1 : 0;
#pragma unroll 1
          for (int n0 = 0; n0 < na; n0 += 16) {
            uint32_t o[16], l[16];
            tmem_ld16(lanes + Z::kO + o_buf * NP + n0, o);
            tmem_ld16(lanes + Z::kL + o_buf * NP + n0, l);
            tmem_ld_wait();
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float d = n0 + r < na ? s_down[n0 + r] : 1.f;
              o[r] = __float_as_uint(__uint_as_float(o[r]) * d);
              l[r] = __float_as_uint(__uint_as_float(l[r]) * d);
            }
            tmem_st16(lanes + Z::kO + o_buf * NP + n0, o);
            tmem_st16(lanes + Z::kL + o_buf * NP + n0, l);
          }
          tmem_st_wait();
        }
      }
      if (i >= 2) ok = await(smem_u32(&pv_done[bf]), ((i >> 1) - 1) & 1, &s_abort) && ok;      // (the MMA that read this P^T)
      uint8_t* const to = s_p + bf * Z::kRowsBytes + p_at;
#pragma unroll 1
      for (int r0 = 0; r0 < na; r0 += 8) {
        float x[8];
        scores(r0, x);
        const float4 h0 = *reinterpret_cast<const float4*>(&s_shift[tb][r0]), h1 = *reinterpret_cast<const float4*>(&s_shift[tb][r0 + 4]);
        const float hs[8] = {h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w};
#pragma unroll
        for (int r = 0; r < 8; ++r)
          *reinterpret_cast<bf16*>(to + (r0 + r) * 128 + ((p_chunk ^ r) << 4)) = __float2bfloat16(ex2(fmaf(x[r], a.scale, hs[r])));
      }
      fence_before();
      fence_async();
      __syncwarp();
      if (lane == 0) { mbar_arrive(smem_u32(&s_free[bf])); mbar_arrive(smem_u32(&p_full[bf])); }
      if (ended_i >= 0) { finish(ended, ended_i, unit - 1, tb == 0 ? 2 : tb - 1, ended_first); ended_i = -1; }
      const Walk here = w;
      begins = next(w);
      if (begins || i + 1 == n) {
        if (Z::kUnits == 2 && i + 1 < n) { ended = here; ended_i = i; ended_first = first; }
        else finish(here, i, unit, tb, first);
        ++unit;
        tb = tb == 2 ? 0 : tb + 1;
        first = 0;
      }
    }
  } else if (warp == 12) {
    // ---- copies.  Of 32 pages each lane holds one's address ----
    int window = -1, id = 0, at_b = -1, unit = 0;
    bool begins = true;
#pragma unroll 1
    for (int i = 0, st = 0, round = 1; i < n; ++i) {
      const int p0 = w.blk * kPages, np = min(kPages, w.pages - p0);
      if (at_b != w.b || window != (p0 & ~31)) {
        at_b = w.b;
        window = p0 & ~31;
        id = a.page_table[size_t(s_seq[w.b]) * a.pages_per_seq + min(window + lane, w.pages - 1)];
      }
      if (i >= kStages) ok = await(smem_u32(&raw_empty[st]), round, &s_abort);
      if (!ok) break;
      const uint32_t bar = smem_u32(&raw_full[st]);
      if (lane == 0) mbar_expect_tx(bar, np * kBlk);
      __syncwarp();
      const int mine = lane - (p0 & 31);
      if (mine >= 0 && mine < np) copy_block(smem_u32(smem) + st * kStage + mine * kBlk, a.pages + (size_t(id) * a.Hkv + w.hk) * kBlk, kBlk, bar);
      if (begins) {                 // Q of the unit
        if (unit >= 2) ok = await(smem_u32(&q_free[unit & 1]), ((unit >> 1) - 1) & 1, &s_abort);
        if (!ok) break;
        uint8_t* const to = s_q + (unit & 1) * Z::kRowsBytes;
        const int na = min(NP, s_nr[w.b] * a.G - w.rt * NP);
#pragma unroll 1
        for (int x0 = 0; x0 < NP * 16; x0 += 128) {      // (zero behind the rows)
          uint4 v[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int x = x0 + 32 * y + lane, r = x >> 4;
            v[y] = make_uint4(0, 0, 0, 0);
            if (r >= na) continue;
            const int row = w.rt * NP + r, vr = verify_row(row);
            v[y] = *reinterpret_cast<const uint4*>(a.q + (size_t(w.b) * a.Rs + vr) * a.ldq + size_t(w.hk * a.G + row - vr * a.G) * kDh + (x & 15) * 8);
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int x = x0 + 32 * y + lane, r = x >> 4, c = x & 15;
            *reinterpret_cast<uint4*>(to + (c >> 3) * (NP * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[y];
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&q_full[unit & 1]));
        ++unit;
      }
      if (++st == kStages) { st = 0; round ^= 1; }
      begins = next(w);
    }
    if (!ok && lane == 0) { const long long t0 = clock64(); while (clock64() - t0 < 2000000) {} }     // (copies in flight land within microseconds)
  } else {
    // ---- MMAs: S of a block, then O of the block before ----
    const uint32_t elected = elect_one();
    const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(NP >> 3) << 17) | (uint32_t(128 >> 4) << 24);
    int unit = 0, before_unit = 0, before_pages = 0;
    bool begins = true, before_begins = false;
#pragma unroll 1
    for (int i = 0; i <= n && ok; ++i) {
      if (i < n) {
        const int bf = i & 1;
        if (begins) ok = await(smem_u32(&q_full[unit & 1]), (unit >> 1) & 1, &s_abort);
        ok = ok && await(smem_u32(&k_full[bf]), (i >> 1) & 1, &s_abort);
        if (ok && i >= 2) ok = await(smem_u32(&s_free[bf]), ((i >> 1) - 1) & 1, &s_abort);
        if (!ok) break;
        fence_after();
        const uint32_t q = smem_u32(s_q + (unit & 1) * Z::kRowsBytes);
        umma_ts4(tmem + Z::kS + bf * NP, tmem + Z::kK + bf * 64, umma_desc(q), idesc, 0, elected);
        umma_ts4(tmem + Z::kS + bf * NP, tmem + Z::kK + bf * 64 + 32, umma_desc(q + NP * 128), idesc, 1, elected);
        umma_commit(smem_u32(&s_full[bf]), elected);
      }
      if (i > 0) {
        const int bf = (i - 1) & 1, o_buf = Z::kUnits == 2 ? before_unit & 1 : 0;
        ok = await(smem_u32(&v_full[bf]), ((i - 1) >> 1) & 1, &s_abort) && await(smem_u32(&p_full[bf]), ((i - 1) >> 1) & 1, &s_abort);
        if (ok && before_begins && before_unit >= Z::kUnits)
          ok = await(smem_u32(&o_free[o_buf]), ((before_unit - Z::kUnits) / Z::kUnits) & 1, &s_abort);
        if (!ok) break;
        fence_after();
        const uint32_t p = smem_u32(s_p + bf * Z::kRowsBytes);
        const uint32_t o_at = tmem + Z::kO + o_buf * NP, l_at = tmem + Z::kL + o_buf * NP, v_at = tmem + Z::kV + bf * 64;
        umma_ts_sums(o_at, l_at, v_at, tmem + Z::kOnes, umma_desc(p), idesc, before_begins ? 0 : 1, min(before_pages, 4), elected);
        if (before_pages > 4) umma_ts_sums(o_at, l_at, v_at + 32, tmem + Z::kOnes, umma_desc(p + NP * 128), idesc, 1, before_pages - 4, elected);
        umma_commit(smem_u32(&pv_done[bf]), elected);
      }
      if (i < n) {
        before_unit = unit; before_begins = begins; before_pages = min(kPages, w.pages - w.blk * kPages);
        begins = next(w);
        if (begins) {
          umma_commit(smem_u32(&q_free[unit & 1]), elected);
          ++unit;
        }
      }
    }
    if (!ok) { const long long t0 = clock64(); while (clock64() - t0 < 2000000) {} }     // (MMAs that are running end within microseconds)
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 13) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  if (s_abort) {
    if (tid == 0) atomicCAS(a.status, 0, LASER_ERR_TIMEOUT);
    return;
  }

  // ---- pieces of units that other CTAs have pieces of, where this is the last of their CTAs ----
  if (s_open[0].b < 0 && s_open[1].b < 0) return;
  if (tid < 2) {
    const Open x = s_open[tid];
    int last = 0;
    if (x.b >= 0) {
      const int before = x.start < 0 ? (per_cta - 1 - x.start) / per_cta : 0, after = (x.start + x.blocks - 1) / per_cta;     // the unit's other CTAs
      __threadfence();
      last = atomicAdd(a.arrived + blockIdx.x - before, 1) == before + after;
      __threadfence();
      if (last) a.arrived[blockIdx.x - before] = 0;
    }
    s_last[tid] = last;
  }
  __syncthreads();
  constexpr int kPer = (NP * 32 + kThreads - 1) / kThreads, kBatch = 4;      // four features of a row: a thread's share
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    if (!s_last[k]) continue;
    const Open x = s_open[k];
    const int before = x.start < 0 ? (per_cta - 1 - x.start) / per_cta : 0, count = before + (x.start + x.blocks - 1) / per_cta + 1;
    // the first CTA's second record, then the others' first ones
    auto record = [&](int r) { return a.part + (2 * size_t(blockIdx.x - before + r) + (r == 0 ? 1 : 0)) * Z::kRecord; };
    const int na = min(NP, s_nr[x.b] * a.G - x.row0);
    float2* const weight = reinterpret_cast<float2*>(smem);                  // [pieces][rows] (m, sum), then (weight, -)
    __syncthreads();
#pragma unroll 1
    for (int y = tid; y < count * NP; y += kThreads)
      if (y % NP < na) weight[y] = __ldcg(reinterpret_cast<const float2*>(record(y / NP) + NP * kDh) + y % NP);
    float4 v[kPer][kBatch], acc[kPer];
    auto fetch = [&](int r0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (r0 + u < count) {
          const float4* rec = reinterpret_cast<const float4*>(record(r0 + u)) + tid;
#pragma unroll
          for (int y = 0; y < kPer; ++y)
            if (tid + y * kThreads < na * 32) v[y][u] = __ldcg(rec + y * kThreads);
        }
    };
    fetch(0);
    __syncthreads();
#pragma unroll 1
    for (int row = warp; row < na; row += kThreads / 32) {
      float top = -INFINITY, sum = 0.f;
      for (int r = lane; r < count; r += 32) top = fmaxf(top, weight[r * NP + row].x);
      for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      for (int r = lane; r < count; r += 32) sum += weight[r * NP + row].y * ex2(weight[r * NP + row].x - top);
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      for (int r = lane; r < count; r += 32) weight[r * NP + row].x = ex2(weight[r * NP + row].x - top) / sum;
    }
    __syncthreads();
#pragma unroll
    for (int y = 0; y < kPer; ++y) acc[y] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int r0 = 0; r0 < count; r0 += kBatch) {
      if (r0) fetch(r0);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (r0 + u >= count) break;
#pragma unroll
        for (int y = 0; y < kPer; ++y) {
          if (tid + y * kThreads >= na * 32) break;
          const float f = weight[(r0 + u) * NP + (tid + y * kThreads) / 32].x;
          acc[y].x += f * v[y][u].x; acc[y].y += f * v[y][u].y; acc[y].z += f * v[y][u].z; acc[y].w += f * v[y][u].w;
        }
      }
    }
#pragma unroll
    for (int y = 0; y < kPer; ++y) {
      const int at = tid + y * kThreads;
      if (at >= na * 32) break;
      const int row = x.row0 + at / 32, r = verify_row(row);
      bf16* to = a.out + (size_t(x.b) * a.Rs + r) * a.ldo + size_t(x.hk * a.G + row - r * a.G) * kDh + (at & 31) * 4;
      *reinterpret_cast<uint32_t*>(to) = pack_bf16(acc[y].x, acc[y].y);
      *reinterpret_cast<uint32_t*>(to + 2) = pack_bf16(acc[y].z, acc[y].w);
    }
  }
}

}  // namespace

size_t attn_int4_wide_part_floats(int ctas) { return size_t(ctas) * 2 * Wide<kMostRows>::kRecord; }

laser_status attn_int4_wide_launch(const AttnArgs& a, int ctas, cudaStream_t stream) {
  const int64_t rows = int64_t(a.Rs) * a.G, tiles = ceil_div(rows, int64_t(kMostRows));
  const int np = int(ceil_div(ceil_div(rows, tiles), int64_t(16))) * 16;
  const int64_t units = a.Hkv * ceil_div(rows, int64_t(np)), blocks = ceil_div(a.pages_per_seq, kPages);     // of a sequence, at most
  if (units * blocks > INT32_MAX) {
    set_error("%lld row tiles a sequence over caches of %d pages are too many for one call", (long long)units, a.pages_per_seq);
    return LASER_ERR_CAPACITY;
  }
  auto launch = [&](auto kernel, int smem) -> laser_status {
    const unsigned grid = unsigned(std::min<int64_t>(ctas, units * a.B * blocks));
    LASER_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    LASER_CUDA(launch_overlapped(kernel, dim3(grid), kThreads, size_t(smem), stream, a));
    return LASER_OK;
  };
  if (np == 16) return launch(attn_int4_wide_kernel<16>, Wide<16>::smem(a.B));
  if (np == 32) return launch(attn_int4_wide_kernel<32>, Wide<32>::smem(a.B));
  return launch(attn_int4_wide_kernel<48>, Wide<48>::smem(a.B));
}

}  // namespace laser
