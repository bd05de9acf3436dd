// Attention of a step's rows over a 4-bit paged cache (int4.cuh): o = sum_t p_t v_t / sum_t p_t, p_t = exp(q . k_t / sqrt(dh)), where row i
// sees the sequence's cached tokens and, of the step's own rows, 0 .. i (chain) or its ancestors and itself (token tree).
//
// The rows of a sequence that share a kv head (rows x n_heads / n_kv_heads) form tiles of 16 - or of 8, where all of them fit that.
// (sequence, kv head, tile) is a unit; all units' pages, one after another, are divided evenly over the SMs (one CTA each) and within a
// CTA over its warps, so ragged lengths leave nobody idle.  A warp walks its pages alone: a page's K and V of a head, codes and scales,
// are one bulk copy into the warp's own ring of shared-memory stages, and the codes become bf16 pairs in registers in the order of the
// MMA's fragments.  16 tokens a step: S = Q K^T and O += P V (tiles of 8 rows: the transposes of both, K and V as the 16-row operand,
// which halves the MMAs), the sum of P as the product with ones.
//
// The softmax's reference m is a whole number in the exponent of two: raising it multiplies p and O by powers of two, exactly, so a
// row's result does not depend on where its walk was cut but for the order of fp32 sums.  It is raised only when a score exceeds it by
// more than 2^6, which a vote finds; p stays below 2^7, and bf16's and fp32's range is left to what is far below.
//
// Where a unit is cut, the pieces (m, sum, O in fp32) meet twice: the warps' in their CTA after its last page, the CTAs' in whichever of
// them arrives last, in the order of the pages both times.  Nothing waits for another CTA.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "int4.cuh"
#include "mma.cuh"
#include "model.cuh"
#include "tma.cuh"
#include "tree.cuh"

namespace laser {
namespace {

using bf16 = __nv_bfloat16;
constexpr int kMaxSeqs = 2048;     // sequences (or prompt chunks) of a call: their offsets are in shared memory
constexpr int kMinPages = 2;       // least pages of a warp: two are in flight together anyway

template <int DH, bool M8>
struct Sizes {
  static constexpr int kWarps = M8 ? 16 : 12;            // 128 or 168 registers a thread
  static constexpr int kStages = DH == 128 ? 4 : 8;
  static constexpr int kRows = M8 ? 8 : 16;
  static constexpr int kBlock = 20 * DH;                 // bytes of a page and head
  static constexpr int kRegs = M8 ? DH / 4 : DH / 2;     // O registers of a lane
  static constexpr int kRecord = (kRegs + 4) * 32;       // floats of a piece: O, m, sums
  static constexpr int kSlice = M8 ? 4 : 8;              // registers that are merged together: neighbouring features
  static constexpr int kSlices = kRegs / kSlice;
  static constexpr int smem(int B) { return kWarps * kStages * (kBlock + 8) + (B + 1) * 16; }
};

struct AttnArgs {
  // rows: from a step's tables (row_ctx, row_n) or the sequences' lengths; parents: a token tree's (up to 64 rows)
  const int32_t *seq_ids, *row_ctx, *row_n, *n_rows, *seq_len, *parents;
  int B, Rs, max_seqs, capacity, Hkv, G;       // G: query heads of a kv head
  const int32_t* page_table;
  int pages_per_seq;
  const uint8_t* pages;                        // this layer's
  const bf16* q;
  bf16* out;
  long long ldq, ldo;                          // elements between rows
  float scale;                                 // log2(e) / sqrt(dh)
  float *part;
  int32_t *arrived, *status;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// two codes at bits 3 .. 6 of the halves -> the two values
__device__ __forceinline__ uint32_t values(uint32_t w, uint32_t s2, uint32_t z2) { return fma2((w & 0x00780078u) | 0x41804180u, s2, z2); }
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void copy_block(uint32_t dst, const void* src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <int N>
__device__ __forceinline__ void lds(uint32_t (&w)[N], const uint8_t* p) {
  if (N == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x; w[1] = u.y; w[2 % N] = u.z; w[3 % N] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x; w[1] = u.y;
  }
}

template <int DH, bool M8>
__global__ void __launch_bounds__(Sizes<DH, M8>::kWarps * 32, 1)
attn_int4_kernel(const AttnArgs a) {
  using Z = Sizes<DH, M8>;
  constexpr int W = Z::kWarps, ST = Z::kStages, TM = Z::kRows, BLK = Z::kBlock;
  constexpr int KW = DH / 32;            // words of a lane's K (of a token) or V (of two tokens)
  constexpr int CPG = DH / 8;            // output features of a lane's column
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* const ring = smem;                                                       // [W][ST][BLK]
  uint64_t* const bars = reinterpret_cast<uint64_t*>(smem + W * ST * BLK);          // [W][ST]
  long long* const s_pre = reinterpret_cast<long long*>(bars + W * ST);             // [B + 1] pages before a sequence
  int* const s_ctx = reinterpret_cast<int*>(s_pre + a.B + 1);                       // [B]
  int* const s_nr = s_ctx + a.B;                                                    // [B]
  __shared__ long long s_sum[W];
  __shared__ int s_abort, s_last[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3;

  next_may_launch();
  if (tid == 0) s_abort = 0;
  if (lane < ST) {
    mbar_init(smem_u32(&bars[warp * ST + lane]), 1);
    mbar_fence_init();
  }
  // a step's tables were complete before any kernel of the forward began
  if (!a.row_ctx) wait_for_earlier();

  // ---- the units: pages of all sequences, one after another ----
  auto tiles_of = [&](int nr) { return (nr * a.G + TM - 1) / TM; };
  long long carry = 0;
  for (int b0 = 0; b0 < a.B; b0 += W * 32) {
    const int b = b0 + tid;
    int ctx = 0, nr = 0;
    if (b < a.B) {
      if (a.row_ctx) {
        ctx = a.row_ctx[b]; nr = a.row_n[b];
      } else {
        const int seq = a.seq_ids[b];
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
      s_ctx[b] = ctx; s_nr[b] = nr;
    }
    const long long mine = nr > 0 ? (long long)a.Hkv * tiles_of(nr) * ((ctx + nr + 15) >> 4) : 0;
    long long x = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) s_sum[warp] = x;
    __syncthreads();
    for (int w = 0; w < warp; ++w) x += s_sum[w];
    if (b < a.B) s_pre[b] = carry + x - mine;
    for (int w = 0; w < W; ++w) carry += s_sum[w];
    __syncthreads();
  }
  if (tid == 0) s_pre[a.B] = carry;
  __syncthreads();
  if (a.row_ctx) wait_for_earlier();
  const long long total = carry;
  const long long per_cta = max((total + gridDim.x - 1) / gridDim.x, (long long)(2 * kMinPages));
  const long long c0 = per_cta * blockIdx.x, c1 = min(total, c0 + per_cta);
  if (c0 >= c1) return;
  const int per_warp = max(int((per_cta + W - 1) / W), kMinPages);
  const long long w0 = c0 + (long long)per_warp * warp;
  const int n = int(max(min(c1 - w0, (long long)per_warp), 0ll));     // this warp's pages

  struct Unit { int b, pages; long long at; };     // a sequence, pages of each of its units, offset of a place in it
  auto find = [&](long long x) {                    // the sequence that page x belongs to
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_pre[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return Unit{lo, (s_ctx[lo] + s_nr[lo] + 15) >> 4, x - s_pre[lo]};
  };
  float* const part = a.part + size_t(blockIdx.x) * (2 * W) * Z::kRecord;                       // the warps' pieces
  float* const cta_part = a.part + (size_t(gridDim.x) * (2 * W) + 2 * blockIdx.x) * Z::kRecord;  // this CTA's

  // a feature pair of a row: the output's place, and its two values
  auto store2 = [&](int b, int hk, int row, int nrows, int feature, float x, float y) {
    if (row < nrows) {
      const int i = row / a.G, j = row % a.G;
      *reinterpret_cast<uint32_t*>(a.out + (size_t(b) * a.Rs + i) * a.ldo + size_t(hk * a.G + j) * DH + feature) = pack_bf16(x, y);
    }
  };

  if (n > 0) {
    uint8_t* const my_ring = ring + warp * ST * BLK;
    const uint32_t ring_at = smem_u32(my_ring), bar_at = smem_u32(bars + warp * ST);
    // ---- copies: a cursor that runs ST pages ahead; 32 page numbers are held, one a lane ----
    Unit u = find(w0);
    int p_b = u.b, p_pages = u.pages, p_unit = int(u.at / u.pages), p_page = int(u.at % u.pages), p_base = -1, p_ids = 0;
    int p_units = a.Hkv * tiles_of(s_nr[p_b]), p_tiles = tiles_of(s_nr[p_b]);
    auto request = [&](int it) {
      if (p_base < 0 || p_page < p_base || p_page >= p_base + 32) {
        p_base = p_page & ~31;
        p_ids = a.page_table[size_t(a.seq_ids[p_b]) * a.pages_per_seq + min(p_base + lane, p_pages - 1)];
      }
      const int phys = __shfl_sync(0xffffffffu, p_ids, p_page - p_base);
      if (lane == 0) {
        const int s = it % ST;
        mbar_expect_tx(bar_at + s * 8, BLK);
        copy_block(ring_at + s * BLK, a.pages + (size_t(phys) * a.Hkv + p_unit / p_tiles) * BLK, BLK, bar_at + s * 8);
      }
      if (++p_page == p_pages) {
        p_page = 0;
        if (++p_unit == p_units) {
          p_unit = 0; p_base = -1;
          do { ++p_b; } while (p_b < a.B && s_nr[p_b] == 0);
          if (p_b < a.B) {
            p_pages = (s_ctx[p_b] + s_nr[p_b] + 15) >> 4;
            p_tiles = tiles_of(s_nr[p_b]);
            p_units = a.Hkv * p_tiles;
          }
        }
      }
    };
    __syncwarp();
    for (int it = 0; it < min(n, ST); ++it) request(it);

    int it = 0, b = u.b, pages = u.pages, tiles = tiles_of(s_nr[b]), unit = int(u.at / u.pages), page = int(u.at % u.pages);
    bool ok = true;
    while (it < n && ok) {
      // ---- a unit, or what of it is this warp's ----
      const int hk = unit / tiles, row0 = (unit % tiles) * TM, nr = s_nr[b], ctx = s_ctx[b], nrows = nr * a.G;
      const int first = page, last = min(pages, page + (n - it));
      // Q: a lane's features are those of its K words
      uint32_t qa[M8 ? 1 : 2][DH / 8];
#pragma unroll
      for (int y = 0; y < (M8 ? 1 : 2); ++y) {
        const int row = row0 + g + 8 * y, i = row / a.G, j = row % a.G;
        const bf16* src = a.q + (size_t(b) * a.Rs + i) * a.ldq + size_t(hk * a.G + j) * DH + qd * (DH / 4);
#pragma unroll
        for (int x = 0; x < DH / 32; ++x) {
          const uint4 v = row < nrows ? reinterpret_cast<const uint4*>(src)[x] : make_uint4(0, 0, 0, 0);
          qa[y][4 * x] = v.x; qa[y][4 * x + 1] = v.y; qa[y][4 * x + 2] = v.z; qa[y][4 * x + 3] = v.w;
        }
      }
      // what the lane's two rows (M8: columns 2 qd, 2 qd + 1) see of the step's own rows: bit j = row j; chains by their last key
      const int ra = min(row0 + (M8 ? 2 * qd : g), nrows - 1) / a.G, rb = min(row0 + (M8 ? 2 * qd + 1 : g + 8), nrows - 1) / a.G;
      unsigned long long see0 = 0, see1 = 0;
      if (a.parents) {
        unsigned long long mask[2];
        tree_paths(a.parents + size_t(b) * a.Rs, nr, lane, mask);
        see0 = tree_path_of(mask, ra);
        see1 = tree_path_of(mask, rb);
      }
      float o[Z::kRegs / 4][4], sums[4] = {0.f, 0.f, 0.f, 0.f}, m[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int t = 0; t < Z::kRegs / 4; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;

      for (; page < last; ++page, ++it) {
        const int s = it % ST;
        if (!mbar_wait_warp(bar_at + s * 8, (it / ST) & 1, &s_abort)) { ok = false; break; }
        const uint8_t* blk = my_ring + s * BLK;
        // ---- scores: M16 sc[0], sc[1] = tokens 0 .. 7, 8 .. 15; M8 sc[0] = even, sc[1] = odd steps of the features ----
        float sc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        {
          uint32_t k0[KW], k1[KW];
          lds<KW>(k0, blk + q4_k_codes(DH, g, qd * KW));
          lds<KW>(k1, blk + q4_k_codes(DH, g + 8, qd * KW));
          const uint32_t sz0 = *reinterpret_cast<const uint32_t*>(blk + q4_k_scale(DH, g, qd * (DH / 4) / 32));
          const uint32_t sz1 = *reinterpret_cast<const uint32_t*>(blk + q4_k_scale(DH, g + 8, qd * (DH / 4) / 32));
          const uint32_t s0 = __byte_perm(sz0, 0, 0x1010), z0 = __byte_perm(sz0, 0, 0x3232);
          const uint32_t s1 = __byte_perm(sz1, 0, 0x1010), z1 = __byte_perm(sz1, 0, 0x3232);
#pragma unroll
          for (int w = 0; w < KW; ++w)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const uint32_t x0 = values(e ? __funnelshift_r(k0[w], k0[w], 8) : k0[w], s0, z0), x1 = values(__funnelshift_r(k0[w], k0[w], 4 * e + 4), s0, z0);
              const uint32_t y0 = values(e ? __funnelshift_r(k1[w], k1[w], 8) : k1[w], s1, z1), y1 = values(__funnelshift_r(k1[w], k1[w], 4 * e + 4), s1, z1);
              const int r = 4 * w + e;
              if (M8) {
                const uint32_t ka[4] = {x0, y0, x1, y1};
                mma16816(sc[e / 2], ka, qa[0][r], qa[0][r + 1]);
              } else {
                const uint32_t qf[4] = {qa[0][r], qa[M8 ? 0 : 1][r], qa[0][r + 1], qa[M8 ? 0 : 1][r + 1]};
                mma16816(sc[0], qf, x0, x1);
                mma16816(sc[1], qf, y0, y1);
              }
            }
        }
        float x[2][4];      // [lane's row][its four tokens], in units of log2
        if (M8) {
#pragma unroll
          for (int c = 0; c < 4; ++c) sc[0][c] += sc[1][c];
        }
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int c = 0; c < 4; ++c) x[y][c] = M8 ? (c < 2 ? sc[0][2 * c + y] : -INFINITY) : sc[c >> 1][2 * y + (c & 1)];
        if (page * 16 + 15 >= ctx) {      // some of the step's own rows, or slots behind them
#pragma unroll
          for (int c = 0; c < (M8 ? 2 : 4); ++c) {
            const int rel = page * 16 + (M8 ? g + 8 * c : (c >> 1) * 8 + 2 * qd + (c & 1)) - ctx;
            if (rel < 0) continue;
            const bool on0 = a.parents ? rel < 64 && (see0 >> (rel & 63) & 1) : rel <= ra;
            const bool on1 = a.parents ? rel < 64 && (see1 >> (rel & 63) & 1) : rel <= rb;
            if (!on0) x[0][c] = -INFINITY;
            if (!on1) x[1][c] = -INFINITY;
          }
        }
        float top[2];
        bool above = false;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          top[y] = M8 ? fmaxf(x[y][0], x[y][1]) : fmaxf(fmaxf(x[y][0], x[y][1]), fmaxf(x[y][2], x[y][3]));
          above = above || top[y] * a.scale > m[y] + 6.f;
        }
        if (__any_sync(0xffffffffu, above)) {
          float down[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float t = top[y];
#pragma unroll
            for (int d = M8 ? 4 : 1; d <= (M8 ? 16 : 2); d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            const float next = fmaxf(m[y], ceilf(t * a.scale));
            down[y] = m[y] == next ? 1.f : ex2(m[y] - next);
            m[y] = next;
          }
#pragma unroll
          for (int t = 0; t < Z::kRegs / 4; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[t][c] *= down[M8 ? c & 1 : c >> 1];
#pragma unroll
          for (int c = 0; c < 4; ++c) sums[c] *= down[M8 ? c & 1 : c >> 1];
        }
        float p[2][4];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float mu = m[y] == -INFINITY ? 0.f : m[y];
#pragma unroll
          for (int c = 0; c < (M8 ? 2 : 4); ++c) p[y][c] = ex2(fmaf(x[y][c], a.scale, -mu));
        }
        // ---- values ----
        {
          uint32_t v0[KW], v1[KW], sz[4];
          lds<KW>(v0, blk + 10 * DH + lane * KW * 4);
          lds<KW>(v1, blk + 10 * DH + (32 + lane) * KW * 4);
          lds<4>(sz, blk + 18 * DH + (g * CPG / 32 * 4 + qd) * 16);
          uint32_t pf[4];
          if (M8) {
            pf[0] = transpose8(pack_bf16(p[0][0], p[1][0]));      // tokens g x rows 2 qd .. -> row g, tokens 2 qd ..
            pf[1] = transpose8(pack_bf16(p[0][1], p[1][1]));
            const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
            mma16816(sums, ones, pf[0], pf[1]);
          } else {
            pf[0] = pack_bf16(p[0][0], p[0][1]);
            pf[1] = pack_bf16(p[1][0], p[1][1]);
            pf[2] = pack_bf16(p[0][2], p[0][3]);
            pf[3] = pack_bf16(p[1][2], p[1][3]);
            mma16816(sums, pf, 0x3f803f80u, 0x3f803f80u);
          }
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            const uint32_t e0 = values(v0[w] << 3, sz[0], sz[1]), f0 = values(v1[w] << 3, sz[2], sz[3]);
            const uint32_t e1 = values(v0[w] >> 1, sz[0], sz[1]), f1 = values(v1[w] >> 1, sz[2], sz[3]);
            const uint32_t e2 = values(v0[w] >> 5, sz[0], sz[1]), f2 = values(v1[w] >> 5, sz[2], sz[3]);
            const uint32_t e3 = values(v0[w] >> 9, sz[0], sz[1]), f3 = values(v1[w] >> 9, sz[2], sz[3]);
            if (M8) {
              const uint32_t va[4] = {e0, e1, f0, f1}, vb[4] = {e2, e3, f2, f3};
              mma16816(o[2 * w], va, pf[0], pf[1]);
              mma16816(o[2 * w + 1], vb, pf[0], pf[1]);
            } else {
              mma16816(o[(4 * w) % (Z::kRegs / 4)], pf, e0, f0);
              mma16816(o[(4 * w + 1) % (Z::kRegs / 4)], pf, e1, f1);
              mma16816(o[(4 * w + 2) % (Z::kRegs / 4)], pf, e2, f2);
              mma16816(o[(4 * w + 3) % (Z::kRegs / 4)], pf, e3, f3);
            }
          }
        }
        __syncwarp();
        if (it + ST < n) request(it + ST);
      }
      if (!ok) break;

      // ---- the unit's result, or the piece that this warp has of it ----
      const int lane_row0 = row0 + (M8 ? 2 * qd : g), lane_row1 = row0 + (M8 ? 2 * qd + 1 : g + 8);
      const float l0 = sums[0], l1 = M8 ? sums[1] : sums[2];
      if (first == 0 && last == pages) {
        const float inv0 = 1.f / l0, inv1 = 1.f / l1;     // (a row sees itself: its sum is not zero)
#pragma unroll
        for (int t = 0; t < Z::kRegs / 4; t += M8 ? 1 : 2) {
          if (M8) {
            store2(b, hk, lane_row0, nrows, CPG * g + 2 * t, o[t][0] * inv0, o[t][2] * inv0);
            store2(b, hk, lane_row1, nrows, CPG * g + 2 * t, o[t][1] * inv1, o[t][3] * inv1);
          } else {
            const int t1 = (t + 1) % (Z::kRegs / 4);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              store2(b, hk, lane_row0, nrows, CPG * (2 * qd + c) + t, o[t][c] * inv0, o[t1][c] * inv0);
              store2(b, hk, lane_row1, nrows, CPG * (2 * qd + c) + t, o[t][2 + c] * inv1, o[t1][2 + c] * inv1);
            }
          }
        }
      } else {
        float* rec = part + (2 * warp + (first == 0 ? 1 : 0)) * Z::kRecord + lane;
#pragma unroll
        for (int t = 0; t < Z::kRegs / 4; ++t)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if ((M8 ? c & 1 : c >> 1) ? lane_row1 < nrows : lane_row0 < nrows) __stcg(rec + (4 * t + c) * 32, o[t][c]);
        __stcg(rec + Z::kRegs * 32, m[0]);
        __stcg(rec + (Z::kRegs + 1) * 32, m[1]);
        __stcg(rec + (Z::kRegs + 2) * 32, l0);
        __stcg(rec + (Z::kRegs + 3) * 32, l1);
      }
      if (page == pages) {
        page = 0;
        if (++unit == a.Hkv * tiles) {
          unit = 0;
          do { ++b; } while (b < a.B && s_nr[b] == 0);
          if (b < a.B) { pages = (s_ctx[b] + s_nr[b] + 15) >> 4; tiles = tiles_of(s_nr[b]); }
        }
      }
    }
    if (!ok && lane == 0)     // copies in flight land before the CTA's memory goes
      for (int x = it; x < min(n, it + ST); ++x) mbar_drain(bar_at + (x % ST) * 8, (x / ST) & 1);
  }
  __syncthreads();
  if (s_abort) {
    if (tid == 0) atomicCAS(a.status, 0, LASER_ERR_TIMEOUT);
    return;
  }

  // ---- pieces: a warp takes slices of the registers, all pieces of them in order ----
  // records first, first + stride, .. (the first one at `first`) -> the output, or a record
  auto merge = [&](const float* head, const float* rest, int count, size_t stride, const Unit& at, float* to) {
    const int nr = s_nr[at.b], tiles = tiles_of(nr), unit = int(at.at / at.pages), hk = unit / tiles, row0 = (unit % tiles) * TM, nrows = nr * a.G;
    const int lane_row0 = row0 + (M8 ? 2 * qd : g), lane_row1 = row0 + (M8 ? 2 * qd + 1 : g + 8);
    for (int sl = warp; sl < Z::kSlices; sl += W) {
      float acc[Z::kSlice], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < Z::kSlice; ++c) acc[c] = 0.f;
#pragma unroll 4
      for (int r = 0; r < count; ++r) {
        const float* rec = (r == 0 ? head : rest + size_t(r - 1) * stride) + lane;
        float v[Z::kSlice], f[2];
#pragma unroll
        for (int c = 0; c < Z::kSlice; ++c) v[c] = __ldcg(rec + (sl * Z::kSlice + c) * 32);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float rm = __ldcg(rec + (Z::kRegs + y) * 32), rl = __ldcg(rec + (Z::kRegs + 2 + y) * 32);
          const float next = fmaxf(m[y], rm);
          const float old = m[y] == next ? 1.f : ex2(m[y] - next);
          f[y] = rm == next ? 1.f : ex2(rm - next);
          if (next == -INFINITY) f[y] = 0.f;        // nothing seen yet
          m[y] = next;
          l[y] = l[y] * old + (f[y] == 0.f ? 0.f : rl * f[y]);
#pragma unroll
          for (int c = 0; c < Z::kSlice; ++c)
            if ((M8 ? c & 1 : c >> 1 & 1) == y) acc[c] = acc[c] * old + (f[y] == 0.f ? 0.f : v[c] * f[y]);
        }
      }
      if (to) {
#pragma unroll
        for (int c = 0; c < Z::kSlice; ++c) __stcg(to + (sl * Z::kSlice + c) * 32 + lane, acc[c]);
        if (sl == 0) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            __stcg(to + (Z::kRegs + y) * 32 + lane, m[y]);
            __stcg(to + (Z::kRegs + 2 + y) * 32 + lane, l[y]);
          }
        }
      } else {
        const float inv0 = 1.f / l[0], inv1 = 1.f / l[1];
        if (M8) {
          store2(at.b, hk, lane_row0, nrows, CPG * g + 2 * sl, acc[0] * inv0, acc[2] * inv0);
          store2(at.b, hk, lane_row1, nrows, CPG * g + 2 * sl, acc[1] * inv1, acc[3] * inv1);
        } else {
          constexpr int H2 = Z::kSlice / 2;      // (the second of two neighbouring features)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            store2(at.b, hk, lane_row0, nrows, CPG * (2 * qd + c) + 2 * sl, acc[c] * inv0, acc[(H2 + c) % Z::kSlice] * inv0);
            store2(at.b, hk, lane_row1, nrows, CPG * (2 * qd + c) + 2 * sl, acc[(2 + c) % Z::kSlice] * inv1, acc[(H2 + 2 + c) % Z::kSlice] * inv1);
          }
        }
      }
    }
  };
  // units with a piece here: those around the CTA's ends and around the places where one warp follows another
  long long done = c0;       // units up to here are dealt with
  long long open_at[2] = {-1, -1};
  for (int w = 0; w * (long long)per_warp < c1 - c0; ++w) {
    const long long begin = c0 + (long long)per_warp * w, end = min(c1, begin + per_warp);
    for (int side = 0; side < 2; ++side) {
      const long long x = side == 0 ? begin : end - 1;      // the warp's first page, and its last
      if (x < done) continue;
      const Unit at = find(x);
      const long long us = x - at.at % at.pages, ue = us + at.pages;
      const long long p0 = max(us, c0), p1 = min(ue, c1);
      done = p1;
      const int f = int((p0 - c0) / per_warp), e = int((p1 - 1 - c0) / per_warp);     // its warps
      const bool open = us < c0 || ue > c1;
      if (f == e && !open) continue;              // one warp had it all
      // a warp's record 0: a piece without the unit's first page
      const float* head = part + (2 * f + (us >= c0 ? 1 : 0)) * Z::kRecord;
      const float* rest = part + (2 * (f + 1)) * Z::kRecord;
      const int which = us < c0 ? 0 : 1;
      merge(head, rest, e - f + 1, size_t(2) * Z::kRecord, at, open ? cta_part + which * Z::kRecord : nullptr);
      if (open) open_at[which] = us;
    }
  }
  if (open_at[0] < 0 && open_at[1] < 0) return;
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    for (int k = 0; k < 2; ++k) {
      s_last[k] = 0;
      if (open_at[k] < 0) continue;
      const Unit at = find(open_at[k]);
      const long long from = open_at[k] / per_cta, to = (open_at[k] + at.pages - 1) / per_cta;     // the unit's CTAs
      if (atomicAdd(a.arrived + from, 1) == int(to - from)) { s_last[k] = 1; a.arrived[from] = 0; }
    }
    __threadfence();
  }
  __syncthreads();
  for (int k = 0; k < 2; ++k) {
    if (!s_last[k]) continue;
    const Unit at = find(open_at[k]);
    const long long from = open_at[k] / per_cta, to = (open_at[k] + at.pages - 1) / per_cta;
    const float* all = a.part + size_t(gridDim.x) * (2 * W) * Z::kRecord;
    merge(all + (2 * from + 1) * Z::kRecord, all + 2 * (from + 1) * Z::kRecord, int(to - from + 1), size_t(2) * Z::kRecord, at, nullptr);
  }
}

laser_status launch_attention(const laser_kv* kv, AttnArgs a, cudaStream_t stream) {
  a.max_seqs = kv->max_seqs;
  a.capacity = int(std::min<int64_t>(kv->capacity_tokens(), INT32_MAX));
  a.Hkv = kv->n_kv_heads; a.G = kv->n_heads / kv->n_kv_heads;
  a.page_table = kv->page_table; a.pages_per_seq = kv->pages_per_seq;
  a.scale = float(1.4426950408889634 / std::sqrt(double(kv->head_dim)));
  a.part = kv->attn_part; a.arrived = kv->attn_arrived;
  auto launch = [&](auto kernel, auto sizes) -> laser_status {
    using Z = decltype(sizes);
    const int smem = Z::smem(a.B);
    const int64_t units = int64_t(a.B) * a.Hkv * ceil_div(a.Rs * a.G, Z::kRows);
    const unsigned grid = unsigned(std::min<int64_t>(kv->attn_ctas, units * kv->pages_per_seq));
    LASER_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    LASER_CUDA(launch_overlapped(kernel, dim3(grid), Z::kWarps * 32, size_t(smem), stream, a));
    return LASER_OK;
  };
  const bool m8 = a.Rs * a.G <= 8;
  if (kv->head_dim == 128) LASER_TRY(m8 ? launch(attn_int4_kernel<128, true>, Sizes<128, true>{}) : launch(attn_int4_kernel<128, false>, Sizes<128, false>{}));
  else LASER_TRY(m8 ? launch(attn_int4_kernel<64, true>, Sizes<64, true>{}) : launch(attn_int4_kernel<64, false>, Sizes<64, false>{}));
  count_launch();
  return LASER_OK;
}

}  // namespace

int attention_int4_max_groups() { return kMaxSeqs; }
size_t attention_int4_part_floats(int head_dim, int ctas) {
  auto of = [&](auto z) { return size_t(ctas) * (2 * decltype(z)::kWarps + 2) * decltype(z)::kRecord; };
  return head_dim == 128 ? std::max(of(Sizes<128, true>{}), of(Sizes<128, false>{})) : std::max(of(Sizes<64, true>{}), of(Sizes<64, false>{}));
}

laser_status attention_int4_launch(laser_model* m, laser_kv* kv, int layer, const int32_t* seq_ids, const int32_t* parents, int B, int Rs,
                                   cudaStream_t stream) {
  AttnArgs a{};
  a.seq_ids = seq_ids; a.row_ctx = m->row_ctx; a.row_n = m->row_n; a.parents = parents;
  a.B = B; a.Rs = Rs;
  a.pages = kv->pages4 + size_t(layer) * kv->layer_bytes4();
  a.q = m->q; a.out = m->attn;
  a.ldq = a.ldo = int64_t(kv->n_heads) * kv->head_dim;
  a.status = m->status;
  return launch_attention(kv, a, stream);
}

}  // namespace laser

using namespace laser;

LASER_API laser_status laser_attend_int4(laser_kv* kv, int32_t layer, const int32_t* seq_ids, const int32_t* parents, const int32_t* n_rows,
                                         int32_t B, int32_t rows, const void* q, int64_t q_stride, void* out, int64_t out_stride, void* stream) {
  LASER_REQUIRE(kv && seq_ids && n_rows && q && out, "null argument");
  LASER_REQUIRE(kv->pages4, "the cache is not a 4-bit one");
  LASER_REQUIRE(layer >= 0 && layer < kv->n_layers, "layer %d out of range", layer);
  LASER_REQUIRE(B >= 0 && rows >= 1 && int64_t(B) * rows <= INT32_MAX, "B = %d sequences of %d rows", B, rows);
  if (B > kMaxSeqs) { set_error("B = %d sequences in one call (at most %d)", B, kMaxSeqs); return LASER_ERR_CAPACITY; }
  LASER_REQUIRE(!parents || rows <= 64, "a token tree has at most 64 rows (rows = %d)", rows);
  const int64_t width = int64_t(kv->n_heads) * kv->head_dim;
  LASER_REQUIRE(q_stride >= width && out_stride >= width, "rows overlap: strides %lld, %lld", (long long)q_stride, (long long)out_stride);
  LASER_REQUIRE((reinterpret_cast<uintptr_t>(q) | uintptr_t(q_stride * 2)) % 16 == 0, "rows of q must be 16-byte aligned");
  LASER_REQUIRE((reinterpret_cast<uintptr_t>(out) | uintptr_t(out_stride * 2)) % 4 == 0, "rows of out must be 4-byte aligned");
  if (B == 0) return LASER_OK;
  AttnArgs a{};
  a.seq_ids = seq_ids; a.n_rows = n_rows; a.seq_len = kv->seq_len; a.parents = parents;
  a.B = B; a.Rs = rows;
  a.pages = kv->pages4 + size_t(layer) * kv->layer_bytes4();
  a.q = static_cast<const __nv_bfloat16*>(q); a.out = static_cast<__nv_bfloat16*>(out);
  a.ldq = q_stride; a.ldo = out_stride;
  a.status = kv->status;
  return launch_attention(kv, a, as_stream(stream));
}
