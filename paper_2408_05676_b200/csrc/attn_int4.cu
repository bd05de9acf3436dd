// Attention of a step's rows over a 4-bit paged cache (int4.cuh): o = sum_t p_t v_t / sum_t p_t, p_t = exp(q . k_t / sqrt(dh)), where row i
// sees the sequence's cached tokens and, of the step's own rows, 0 .. i (chain) or its ancestors and itself (token tree).
//
// The rows of a sequence that share a kv head (rows x n_heads / n_kv_heads) form tiles of 8 NT rows, NT = 1 .. 5.  (sequence, kv head,
// tile) is a unit; all units' pages, one after another, are divided evenly over the SMs (one CTA each) and within a CTA over its teams, so
// ragged lengths leave nobody idle.  A team is a warp, or two where NT > 1.  It walks its pages alone: a page's K and V of a head, codes
// and scales, come by 16-byte copies into the warp's own ring of shared-memory stages (a bulk copy and its barrier cost a warp 300 clocks
// a page, these 100), and the codes become bf16 pairs in registers in the order of the MMA's fragments.  S^T = K Q^T and O^T += V^T P^T:
// tokens and features are the 16-row operand, so that what was unpacked serves all of the tile's rows, eight at a time, and few rows waste
// little.  The sum of P is the product with ones.  Of a team's two warps each takes one page of two, then both pages' P and half of the
// features: half the registers of O a lane, and no page is unpacked twice (one text of 64 thousand tokens, 36 rows: 56 us instead of 66).
//
// What bounds it: the instructions.  A warp-level MMA of 16 x 8 x 16 keeps a scheduler from issuing for eight clocks; a page is 16 NT of
// them, and some 350 other instructions, 200 of them to unpack 4096 codes.  One row at a time over long texts reads 5.0 TB/s of the 6.6 that
// a copy reaches; 17 rows take 940 clocks a page and scheduler.  On tensor memory, whose MMAs issue once for 128 tokens, the hand-overs
// between unpacking, products and softmax took longer than what they saved (17 rows: 205 us instead of 122; 36 rows: 69 instead of 52).
//
// The softmax's reference m is a whole number in the exponent of two: raising it multiplies p and O by powers of two, exactly, so a
// row's result does not depend on where its walk was cut but for the order of fp32 sums.  It is raised only when a score exceeds it by
// more than 2^6, which a vote finds; p stays below 2^7, and bf16's and fp32's range is left to what is far below.
//
// Where a unit is cut, the pieces (m, sum, O in fp32) meet twice, in the order of the pages both times: the teams' in their CTA after its
// last page, the CTAs' in a kernel that follows.
//
// Times (us; floors by bytes at 6.56 TB/s in brackets): 32 heads of 128, 9 rows over one text of 512 tokens 9.1 (0.4), over 16 of 256 to 768
// 21.4 (6.7); 40 heads, trees of 17 rows over 64 texts of 256 to 1024 122 (42); 32 heads of 8 kv heads, one row over 64 texts of 4096 to 8192
// 101 (77), 9 rows over one of 65536 52 (13).
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
constexpr int kMaxSeqs = 1024;     // sequences (or prompt chunks) of a call: their offsets are in shared memory
constexpr int kMostTiles = 5;      // of eight rows in a tile: O takes 80 registers then (of three at most, 36 rows' pages are unpacked twice: 71 us instead of 69)

// a unit that several CTAs have pieces of (count = 0: none)
struct Join { int b, hk, row0, rows, count; };

template <int DH, int NT>
struct Sizes {
  // A team is a warp, or two that take a page each of every two and half of the features each (one row over long texts: 100 us alone, 112 in
  // twos; 36 rows: 66 alone, 52 in twos)
  static constexpr int kTeam = NT == 1 ? 1 : 2;
  static constexpr int kRegsO = NT * DH / 4 / kTeam;     // O registers of a lane
  // as many warps as the registers allow without spills (heads of 64, 9 rows: 55 us with 16, 58 with 12, 71 with 8; of 128, 17 rows: 157 with 16
  // and spills, 121 with 12, 137 with 8; 36 rows: 65 with 12 and spills, 52 with 8)
  static constexpr int kWarps = NT == 1 || kRegsO <= 24 ? 16 : kRegsO <= 48 ? 12 : 8;
  static constexpr int kTeams = kWarps / kTeam;
  static constexpr int kRows = 8 * NT;
  static constexpr int kBlock = q4_block_bytes(DH);      // bytes of a page and head
  static constexpr int kStages = kTeam == 1 ? 4 : 3;     // of a warp's ring (one more: no change)
  static constexpr bool kQInSmem = NT > 1;               // each lane's share of Q is put by and read again for every page
  static constexpr int kQBytes = kQInSmem ? NT * DH / 8 * 4 * 32 : 0;
  static constexpr int kPBytes = kTeam == 1 ? 0 : NT * 2 * 256;          // P of two pages
  static constexpr int kSlices = NT * DH / 16;           // of O: four registers, two neighbouring features of two rows
  static constexpr int kOBytes = kSlices * 512;          // O of a piece
  // A team's memory: its rings, Q and P; when those are done with, O of the piece that it ends with and slices of others' first pieces
  static constexpr int kLoop = kTeam * kStages * kBlock + kQBytes + 2 * kPBytes;
  static constexpr int kFetched = kTeam == 1 ? 16 : 8;   // slices of a warp
  static constexpr int kRegion = kLoop > kOBytes + kTeam * kFetched * 512 ? kLoop : kOBytes + kTeam * kFetched * 512;
  static constexpr int kRecord = kOBytes / 4 + 16 * NT;  // floats of a CTA's piece: O, then (m, sum) of the rows
  static constexpr int smem(int B) { return kTeams * kRegion + (B + 1) * 8 + B * 12; }
  static constexpr int kPart = kTeams * (kOBytes / 4);   // floats of a CTA's teams' first pieces
  static size_t part_floats(int ctas) { return size_t(ctas) * (kPart + 2 * kRecord) + size_t(ctas) * (sizeof(Join) / 4); }
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
  int vec_out;                                 // rows of out are 16-byte aligned
  unsigned group_inv;                          // 2^32 / G rounded up (G > 1)
  float scale;                                 // log2(e) / sqrt(dh)
  float *part, *records;                       // warps' first pieces; CTAs' pieces [CTA][2]: of the unit that it goes on with, that goes on behind it
  Join* joins;                                 // [CTA] the latter
  int32_t* status;
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
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// two codes at bits 3 .. 6 of the halves -> the two values.  (w & 0x00780078) | 0x41804180 as one instruction: of two constants the
// compiler makes two, and the kernel's busiest pipe is the one for logic and shifts.
__device__ __forceinline__ uint32_t values(uint32_t w, uint32_t s2, uint32_t z2) {
  uint32_t u;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(w), "r"(0x00780078u), "r"(0x41804180u));
  return fma2(u, s2, z2);
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void lds(uint32_t (&w)[N], const uint8_t* p) {
  if (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if (N == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x; w[1 % N] = u.y; w[2 % N] = u.z; w[3 % N] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x; w[1 % N] = u.y;
  }
}

// of two warps: all have come here; whether any thread says so
__device__ __forceinline__ void team_sync(int team) { asm volatile("bar.sync %0, 64;" ::"r"(1 + team) : "memory"); }
__device__ __forceinline__ bool team_any(int team, bool x) {
  uint32_t y;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbar.red.or.pred q, %2, 64, p;\nselp.u32 %0, 1, 0, q;\n}"
               : "=r"(y) : "r"(uint32_t(x)), "r"(1 + team) : "memory");
  return y != 0;
}

// a unit: its sequence, kv head and first row; its first block (from the CTA's first) and its blocks
struct Segment { int b, hk, row0, start, blocks; };
// one that is cut: the teams whose pieces are this CTA's; whether the last of them went on behind it; whether other CTAs have pieces, and
// then whether they have its beginning
struct Cut { Segment seg; int first, last; bool early, open, begun; };
// -m of rows that have seen nothing: above every score x scale that 32 bits hold (6.1e37), so that the first score a row sees, however low,
// gives it a reference
constexpr float kNothing = 1e38f;

// ceil(total / parts), parts below 2^16; in 32 bits where they hold total + parts (in 64 a division takes 100 instructions)
__host__ __device__ constexpr int share_of(long long total, unsigned parts) {
  return total <= 0xffffffffll - 0xffff ? int((unsigned(total) + parts - 1) / parts) : int((total + parts - 1) / parts);
}
static_assert(share_of(0xffffffffll, 148) == 29020050 && share_of(0xffffffffll - 0xffff, 148) == 29019607 && share_of(0x100000000ll, 148) == 29020050 &&
              share_of(149, 148) == 2 && share_of(1, 148) == 1, "");

template <int DH, int NT>
__global__ void __launch_bounds__(Sizes<DH, NT>::kWarps * 32, 1)
attn_int4_kernel(const AttnArgs a) {
  using Z = Sizes<DH, NT>;
  constexpr int S = Z::kTeam, W = Z::kWarps, T = Z::kTeams, ST = Z::kStages, TM = Z::kRows, BLK = Z::kBlock;
  constexpr int KW = DH / 32;            // words of a lane's K (of a token) or V (of two tokens)
  constexpr int VW = KW / S;             // of V, a warp's
  constexpr int CPG = DH / 8;            // output features of a lane
  constexpr int MT = DH / 16;            // 16-feature tiles
  constexpr int OT = MT / S;             // a warp's
  constexpr int QC = DH / 32;            // 16-byte pieces of a lane's share of a Q row
  extern __shared__ __align__(128) uint8_t smem[];
  long long* const s_pre = reinterpret_cast<long long*>(smem + T * Z::kRegion);     // [B + 1] blocks before a sequence, behind the teams' regions
  int* const s_ctx = reinterpret_cast<int*>(s_pre + a.B + 1);                       // [B]
  int* const s_nr = s_ctx + a.B;                                                    // [B]
  int* const s_seq = s_nr + a.B;                                                    // [B]
  __shared__ long long s_sum[W];
  __shared__ unsigned long long s_path[T][64];      // token trees: the rows that a row of the team's sequence sees
  __shared__ Segment s_seg[T][2];                   // the units of a team's first and of its last block
  __shared__ Cut s_cut[2 * T];
  __shared__ __align__(16) float2 s_ml[T][2][TM];   // m and sum of the rows of the piece that a team began with, if it went on; that it ended with
  __shared__ float s_half[S == 1 ? 1 : W][TM];      // what a warp tells the other of its rows: highest scores, or sums
  __shared__ int s_cuts;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3, team = warp / S, half = warp % S;
  // a row is verify row row / G, head row % G of its kv head
  auto verify_row = [&](int row) { return a.G == 1 ? row : int(__umulhi(unsigned(row), a.group_inv)); };

  next_may_launch();
  // a step's tables were complete before any kernel of the forward began
  if (!a.row_ctx) wait_for_earlier();

  // ---- the units: blocks of S pages of all sequences, one after another ----
  auto tiles_of = [&](int nr) { return (nr * a.G + TM - 1) / TM; };
  auto pages_of = [&](int b) { return (s_ctx[b] + s_nr[b] + 15) >> 4; };
  long long total = 0;
  for (int b0 = 0; b0 < a.B; b0 += W * 32) {
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
    const long long mine = nr > 0 ? (long long)(a.Hkv * tiles_of(nr)) * ((((ctx + nr + 15) >> 4) + S - 1) / S) : 0;
    long long x = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) s_sum[warp] = x;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w == warp) x += all;
      all += s_sum[w];
    }
    if (b < a.B) s_pre[b] = total + x - mine;
    total += all;
    __syncthreads();
  }
  if (a.row_ctx) wait_for_earlier();
  // (below 2^31: launch_attention sees to it)
  constexpr int kLeast = 2 / S;        // blocks of a team: two pages are in flight together anyway
  const int per_cta = max(share_of(total, gridDim.x), 2 * kLeast);
  const long long c0 = (long long)per_cta * blockIdx.x;
  if (tid == 0) a.joins[blockIdx.x].count = 0;
  if (c0 >= total) return;
  const int span = int(min(total - c0, (long long)per_cta));      // this CTA's blocks
  const int per_team = max((per_cta + T - 1) / T, kLeast);
  const int n = min(span - per_team * team, per_team);            // this team's (none, if that is negative)

  float4* const my_part = reinterpret_cast<float4*>(a.part) + size_t(blockIdx.x * T + team) * (Z::kSlices * 32) + lane;   // the team's first piece

  if (n > 0) {
    uint8_t* const region = smem + team * Z::kRegion;
    const uint32_t ring_at = smem_u32(region) + half * (ST * BLK) + lane * 16;
    // ---- where the team begins ----
    int b, tile, hk, blk;
    {
      const long long x = c0 + per_team * team;
      int lo = 0, hi = a.B - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_pre[mid] <= x) lo = mid; else hi = mid - 1;
      }
      b = lo;
      const unsigned at = unsigned(x - s_pre[b]), of = unsigned(pages_of(b) + S - 1) / S, unit = at / of, tl = unsigned(tiles_of(s_nr[b]));
      blk = int(at - unit * of); hk = int(unit / tl); tile = int(unit - hk * tl);
    }
    int pages = pages_of(b), blocks = (pages + S - 1) / S, tiles = tiles_of(s_nr[b]);

    // ---- copies: a cursor that runs ST blocks ahead; of 32 pages each lane holds one's number ----
    int p_b = b, p_tile = tile, p_hk = hk, p_page = blk * S + half, p_pages = pages, p_tiles = tiles, p_stop = 0, p_window = -1, p_id = 0;
    auto aim = [&]() {
      if (p_window != (p_page & ~31)) {
        p_window = p_page & ~31;
        p_id = a.page_table[size_t(s_seq[p_b]) * a.pages_per_seq + min(p_window + lane, p_pages - 1)];
      }
      p_stop = min(p_pages, p_window + 32);
    };
    auto request = [&](int s) {
      const int id = __shfl_sync(0xffffffffu, p_id, p_page & 31);
      if (S == 1 || p_page < p_pages) {          // (not so where a unit's pages are odd)
        const uint8_t* src = a.pages + (size_t(id) * a.Hkv + p_hk) * BLK + lane * 16;
#pragma unroll
        for (int x = 0; x + 512 <= BLK; x += 512) copy16(ring_at + s * BLK + x, src + x);
        if (BLK % 512 && lane < BLK % 512 / 16) copy16(ring_at + s * BLK + BLK / 512 * 512, src + BLK / 512 * 512);
      }
      p_page += S;
      if (p_page - half < p_stop) return;
      if (p_page - half >= p_pages) {
        p_page = half;
        if (++p_tile == p_tiles) {
          p_tile = 0;
          if (++p_hk == a.Hkv) {
            p_hk = 0;
            do { ++p_b; } while (p_b < a.B && s_nr[p_b] == 0);
            if (p_b >= a.B) return;             // (the last page of all: nothing is requested after it)
            p_window = -1;
            p_pages = pages_of(p_b);
            p_tiles = tiles_of(s_nr[p_b]);
          }
        }
      }
      aim();
    };
    __syncwarp();
    aim();
#pragma unroll 1
    for (int s = 0; s < ST; ++s) {
      if (s < n) request(s);
      copies_end();
    }

    int it = 0, path_b = -1, stage = 0;
    while (it < n) {
      // ---- a unit, or what of it is this team's ----
      const int row0 = tile * TM, nr = s_nr[b], ctx = s_ctx[b], nrows = nr * a.G;
      const int first = blk, last = min(blocks, blk + (n - it));
      if (half == 0 && lane == 0) {
        const Segment seg{b, hk, row0, per_team * team + it - blk, blocks};
        if (it == 0) s_seg[team][0] = seg;
        if (n - it <= blocks - blk) s_seg[team][1] = seg;
      }
      // Q: a lane's features are those of its K words
      uint32_t qa[Z::kQInSmem ? 1 : DH / 8];
      uint4* const my_q = reinterpret_cast<uint4*>(region + S * ST * BLK) + lane;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int row = row0 + 8 * t + g, i = verify_row(row), j = row - i * a.G;
        const bf16* src = a.q + (size_t(b) * a.Rs + i) * a.ldq + size_t(hk * a.G + j) * DH + qd * (DH / 4);
#pragma unroll
        for (int y = 0; y < QC / S; ++y) {
          const int x = half * (QC / S) + y;
          const uint4 v = row < nrows ? reinterpret_cast<const uint4*>(src)[x] : make_uint4(0, 0, 0, 0);
          if (Z::kQInSmem) {
            my_q[(t * QC + x) * 32] = v;
          } else {
            uint32_t* to = qa + (Z::kQInSmem ? 0 : 4 * x);
            to[0] = v.x; to[Z::kQInSmem ? 0 : 1] = v.y; to[Z::kQInSmem ? 0 : 2] = v.z; to[Z::kQInSmem ? 0 : 3] = v.w;
          }
        }
      }
      if (a.parents && path_b != b) {
        if (half == 0) {
          unsigned long long mask[2];
          tree_paths(a.parents + size_t(b) * a.Rs, nr, lane, mask);
          __syncwarp();
          s_path[team][lane] = mask[0];
          s_path[team][lane + 32] = mask[1];
          __syncwarp();
        }
        path_b = b;
      }
      if (S == 2) team_sync(team);
      // shift = -m, with m the softmax's reference: p = 2^(score x scale + shift)
      float o[NT][OT][4], sums[NT][4], shift[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        shift[t][0] = shift[t][1] = kNothing;
        sums[t][0] = sums[t][1] = sums[t][2] = sums[t][3] = 0.f;
#pragma unroll
        for (int f = 0; f < OT; ++f) o[t][f][0] = o[t][f][1] = o[t][f][2] = o[t][f][3] = 0.f;
      }

#pragma unroll 1
      for (; blk < last; ++blk, ++it) {
        copies_but<ST - S>();
        __syncwarp();
        const uint8_t* mine = region + (half * ST + stage) * BLK;
        // ---- scores: of tokens g and g + 8 (the halves of x) and the lane's rows 2 qd, 2 qd + 1 of each tile ----
        float x[NT][4];
        {
#pragma unroll
          for (int t = 0; t < NT; ++t) x[t][0] = x[t][1] = x[t][2] = x[t][3] = 0.f;
          uint32_t k0[KW], k1[KW];
          lds<KW>(k0, mine + q4_k_codes(DH, g, qd * KW));
          lds<KW>(k1, mine + q4_k_codes(DH, g + 8, qd * KW));
          const uint32_t sz0 = *reinterpret_cast<const uint32_t*>(mine + q4_k_scale(DH, g, qd * (DH / 4) / 32));
          const uint32_t sz1 = *reinterpret_cast<const uint32_t*>(mine + q4_k_scale(DH, g + 8, qd * (DH / 4) / 32));
          const uint32_t s0 = __byte_perm(sz0, 0, 0x1010), z0 = __byte_perm(sz0, 0, 0x3232);
          const uint32_t s1 = __byte_perm(sz1, 0, 0x1010), z1 = __byte_perm(sz1, 0, 0x3232);
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            const uint32_t ka[4] = {values(k0[w], s0, z0), values(k1[w], s1, z1), values(__funnelshift_r(k0[w], k0[w], 4), s0, z0),
                                    values(__funnelshift_r(k1[w], k1[w], 4), s1, z1)};
            const uint32_t kb[4] = {values(__funnelshift_r(k0[w], k0[w], 8), s0, z0), values(__funnelshift_r(k1[w], k1[w], 8), s1, z1),
                                    values(__funnelshift_r(k0[w], k0[w], 12), s0, z0), values(__funnelshift_r(k1[w], k1[w], 12), s1, z1)};
            uint4 q[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const uint32_t* own = qa + (Z::kQInSmem ? 0 : 4 * w);
              q[t] = Z::kQInSmem ? my_q[(t * QC + w) * 32] : make_uint4(own[0], own[Z::kQInSmem ? 0 : 1], own[Z::kQInSmem ? 0 : 2], own[Z::kQInSmem ? 0 : 3]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816(x[t], ka, q[t].x, q[t].y);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816(x[t], kb, q[t].z, q[t].w);
          }
        }
        const int page = blk * S + half;        // (the second of a team's may be one too many: all of it is masked)
        if (page * 16 + 15 >= ctx) {            // some of the step's own rows, or slots behind them
          const int rel0 = page * 16 + g - ctx, rel1 = rel0 + 8;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int i = verify_row(min(row0 + 8 * t + 2 * qd + y, nrows - 1));      // (rows that are not active: as the last)
              if (a.parents) {
                const unsigned long long see = s_path[team][i];
                if (rel0 >= 0 && (rel0 >= 64 || !(see >> (rel0 & 63) & 1))) x[t][y] = -INFINITY;
                if (rel1 >= 0 && (rel1 >= 64 || !(see >> (rel1 & 63) & 1))) x[t][2 + y] = -INFINITY;
              } else {
                if (rel0 > i) x[t][y] = -INFINITY;
                if (rel1 > i) x[t][2 + y] = -INFINITY;
              }
            }
        }
        // probabilities: from (token, row) to the second product's fragments, a row's tokens 2 qd, 2 qd + 1 (and 8 on) in lane g
        uint32_t p[NT][2];
        uint2* const team_p = reinterpret_cast<uint2*>(region + S * ST * BLK + Z::kQBytes + (it & 1) * Z::kPBytes) + lane;
        // The reference came of a product rounded to 32 bits, so the products are rounded, too, before it is added: in one step (2 % less for one
        // row's time over long texts) what that rounding dropped would be left as an exponent, without bound where scores are above 2^24.
        auto exponent = [&](int t, int c) { return __fadd_rn(__fmul_rn(x[t][c], a.scale), shift[t][c & 1]); };
        auto probabilities = [&]() {        // whether one is above 2^6
          uint32_t highest = 0;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            p[t][0] = pack_bf16(ex2(exponent(t, 0)), ex2(exponent(t, 1)));
            p[t][1] = pack_bf16(ex2(exponent(t, 2)), ex2(exponent(t, 3)));
            highest = max2(highest, max2(p[t][0], p[t][1]));
            p[t][0] = transpose8(p[t][0]);
            p[t][1] = transpose8(p[t][1]);
            if (S == 2) team_p[(half * NT + t) * 32] = make_uint2(p[t][0], p[t][1]);
          }
          return max2(highest, 0x42804280u) != 0x42804280u;
        };
        // (with the reference as it is; again if that turns out too low)
        const bool above = probabilities();
        if (S == 1 ? __any_sync(0xffffffffu, above) : team_any(team, above)) {
          float top[NT][2];
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              top[t][y] = fmaxf(x[t][y], x[t][2 + y]);
#pragma unroll
              for (int d = 4; d <= 16; d <<= 1) top[t][y] = fmaxf(top[t][y], __shfl_xor_sync(0xffffffffu, top[t][y], d));
              if (S == 2 && g == 0) s_half[S == 1 ? 0 : warp][8 * t + 2 * qd + y] = top[t][y];
            }
          if (S == 2) team_sync(team);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            float down[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              if (S == 2) top[t][y] = fmaxf(top[t][y], s_half[S == 1 ? 0 : warp ^ 1][8 * t + 2 * qd + y]);
              const float next = fminf(shift[t][y], -ceilf(__fmul_rn(top[t][y], a.scale)));
              down[y] = ex2(next - shift[t][y]);
              shift[t][y] = next;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) sums[t][c] *= down[c & 1];
#pragma unroll
            for (int f = 0; f < OT; ++f)
#pragma unroll
              for (int c = 0; c < 4; ++c) o[t][f][c] *= down[c & 1];
          }
          probabilities();
          if (S == 2) team_sync(team);
        }
        // (with that vote both are done with the block before)
        if (S == 2 && it > 0) {
          if (it - 1 + ST < n) request(stage == 0 ? ST - 1 : stage - 1);
          copies_end();
        }
        const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int t = 0; t < NT; ++t) mma16816(sums[t], ones, p[t][0], p[t][1]);
        // ---- values ----
#pragma unroll
        for (int h = 0; h < S; ++h) {
          if (h == 1 && 2 * blk + 1 >= pages) break;
          const uint8_t* from = region + (h * ST + stage) * BLK;
          uint32_t v0[VW], v1[VW], sz[4];
          lds<VW>(v0, from + 10 * DH + lane * KW * 4 + half * VW * 4);
          lds<VW>(v1, from + 10 * DH + (32 + lane) * KW * 4 + half * VW * 4);
          lds<4>(sz, from + 18 * DH + (g * CPG / 32 * 4 + qd) * 16);
          if (S == 2) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const uint2 u = team_p[(h * NT + t) * 32];
              p[t][0] = u.x; p[t][1] = u.y;
            }
          }
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            const uint32_t va[4] = {values(v0[w] << 3, sz[0], sz[1]), values(v0[w] >> 1, sz[0], sz[1]), values(v1[w] << 3, sz[2], sz[3]),
                                    values(v1[w] >> 1, sz[2], sz[3])};
            const uint32_t vb[4] = {values(v0[w] >> 5, sz[0], sz[1]), values(v0[w] >> 9, sz[0], sz[1]), values(v1[w] >> 5, sz[2], sz[3]),
                                    values(v1[w] >> 9, sz[2], sz[3])};
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816(o[t][2 * w], va, p[t][0], p[t][1]);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816(o[t][2 * w + 1], vb, p[t][0], p[t][1]);
          }
        }
        if (S == 1) {
          __syncwarp();
          if (it + ST < n) request(stage);
          copies_end();
        }
        if (++stage == ST) stage = 0;
      }

      // ---- the unit's result, or the piece that this team has of it ----
      if (S == 2) {                            // the sums: each warp's pages'
        if (g == 0) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int y = 0; y < 2; ++y) s_half[S == 1 ? 0 : warp][8 * t + 2 * qd + y] = sums[t][y];
        }
        team_sync(team);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int y = 0; y < 2; ++y) sums[t][y] += s_half[S == 1 ? 0 : warp ^ 1][8 * t + 2 * qd + y];
      }
      if (first == 0 && last == blocks) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int row = row0 + 8 * t + 2 * qd + y;
            if (row >= nrows) continue;
            const float inv = 1.f / sums[t][y];      // (a row sees itself: its sum is not zero)
            const int i = verify_row(row), j = row - i * a.G;
            bf16* dst = a.out + (size_t(b) * a.Rs + i) * a.ldo + size_t(hk * a.G + j) * DH + CPG * g + 2 * OT * half;
            uint32_t w[OT];
#pragma unroll
            for (int f = 0; f < OT; ++f) w[f] = pack_bf16(o[t][f][y] * inv, o[t][f][2 + y] * inv);
            if (a.vec_out && OT >= 4) {
#pragma unroll
              for (int f = 0; f < OT; f += 4) *reinterpret_cast<uint4*>(dst + 2 * f) = make_uint4(w[f], w[(f + 1) % OT], w[(f + 2) % OT], w[(f + 3) % OT]);
            } else {
#pragma unroll
              for (int f = 0; f < OT; ++f) *reinterpret_cast<uint32_t*>(dst + 2 * f) = w[f];
            }
          }
      } else {
        const bool early = it < n;      // the team goes on: its memory is not free yet
        __syncwarp();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (row0 + 8 * t >= nrows) break;      // (no row of the tile)
#pragma unroll
          for (int f = 0; f < OT; ++f) {
            const float4 v = make_float4(o[t][f][0], o[t][f][1], o[t][f][2], o[t][f][3]);
            const int sl = t * MT + half * OT + f;
            if (early) __stcg(my_part + sl * 32, v);
            else reinterpret_cast<float4*>(region)[sl * 32 + lane] = v;
          }
          if (half == 0 && g == 0) {
#pragma unroll
            for (int y = 0; y < 2; ++y) s_ml[team][early ? 0 : 1][8 * t + 2 * qd + y] = make_float2(shift[t][y] == kNothing ? -INFINITY : -shift[t][y], sums[t][y]);
          }
        }
      }
      if (blk == blocks) {
        blk = 0;
        if (++tile == tiles) {
          tile = 0;
          if (++hk == a.Hkv) {
            hk = 0;
            do { ++b; } while (b < a.B && s_nr[b] == 0);
            if (b < a.B) { pages = pages_of(b); blocks = (pages + S - 1) / S; tiles = tiles_of(s_nr[b]); }
          }
        }
      }
    }
  }
  __syncthreads();

  // ---- this CTA's pieces: of units around its ends and around the places where one team follows another ----
  if (warp == 0) {
    const int w = lane >> 1, begin_w = w * per_team;
    Cut c{};
    bool here = lane < 2 * T && begin_w < span;
    if (here) {
      c.seg = s_seg[w][lane & 1];
      const int end = c.seg.start + c.seg.blocks;
      here = lane == 0 || s_seg[(lane - 1) >> 1][(lane - 1) & 1].start != c.seg.start;        // (the first to list it)
      c.first = w;
      c.last = (min(end, span) - 1) / per_team;
      c.begun = c.seg.start < 0;
      c.open = c.begun || end > span;
      c.early = end < min((c.last + 1) * per_team, span);
      here = here && (c.open || c.first != c.last);       // (else one team had it all)
    }
    const unsigned all = __ballot_sync(0xffffffffu, here);
    if (here) s_cut[__popc(all & ((1u << lane) - 1))] = c;
    if (lane == 0) s_cuts = __popc(all);
  }
  __syncthreads();
  const int cuts = s_cuts;
  // Four slices of eight rows at a time, the warps in turn.  First pieces' come from L2, as many together as there is room for.
  constexpr int kParts = Z::kSlices / 4, kTogether = Z::kFetched / 4;
  const int mine = (cuts * kParts - warp + W - 1) / W;
  float4* const fetched = reinterpret_cast<float4*>(smem + team * Z::kRegion + Z::kOBytes + half * (Z::kFetched * 512)) + lane;
  auto fetch = [&](int x0) {
#pragma unroll 1
    for (int x = x0; x < min(x0 + kTogether, mine); ++x) {
      const int c = (warp + x * W) / kParts, part = warp + x * W - c * kParts;
      if (!s_cut[c].early) continue;
      const float4* from = reinterpret_cast<const float4*>(a.part) + (size_t(blockIdx.x * T + s_cut[c].last) * Z::kSlices + 4 * part) * 32 + lane;
#pragma unroll
      for (int k = 0; k < 4; ++k) copy16(smem_u32(fetched + ((x - x0) * 4 + k) * 32), from + k * 32);
    }
  };
  fetch(0);
  // what each piece of a row counts, in the place of its m; of a unit that other CTAs have pieces of, m and the sum go with this one's
  auto record = [&](const Cut& c) { return a.records + size_t(2 * blockIdx.x + (c.begun ? 0 : 1)) * Z::kRecord; };
#pragma unroll 1
  for (int y = tid; y < cuts * TM; y += W * 32) {
    const Cut& c = s_cut[y / TM];
    const int row = y % TM, first = c.first, last = c.last, at_end = c.early ? last : -1;
    float2 ml[T];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < T; ++x) {
      ml[x] = x >= first && x <= last ? s_ml[x][x == at_end ? 0 : 1][row] : make_float2(-INFINITY, 0.f);
      m = fmaxf(m, ml[x].x);
    }
    const float zero = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int x = 0; x < T; ++x) {
      ml[x].x = ex2(ml[x].x - zero);
      l += ml[x].y * ml[x].x;
    }
    if (c.open) __stcg(reinterpret_cast<float2*>(record(c) + Z::kOBytes / 4) + row, make_float2(m, l));
    const float by = c.open ? 1.f : 1.f / l;
#pragma unroll
    for (int x = 0; x < T; ++x)
      if (x >= first && x <= last) s_ml[x][x == at_end ? 0 : 1][row].x = ml[x].x * by;
  }
  __syncthreads();
#pragma unroll 1
  for (int x0 = 0; x0 < mine; x0 += kTogether) {
    if (x0) fetch(x0);
    copies_done();                                // (a lane reads what it fetched itself)
#pragma unroll 1
    for (int x = x0; x < min(x0 + kTogether, mine); ++x) {
      const int at = (warp + x * W) / kParts, part = warp + x * W - at * kParts, t = part / (MT / 4), f = part % (MT / 4) * 4;
      const Cut& c = s_cut[at];
      const int first = c.first, last = c.last, nrows = s_nr[c.seg.b] * a.G;
      const bool early = c.early;
      if (c.seg.row0 + 8 * t >= nrows) continue;
      float acc[4][4] = {};
      const float4* o = reinterpret_cast<const float4*>(smem + first * Z::kRegion) + part * 128 + lane;
      const float4* w = reinterpret_cast<const float4*>(&s_ml[first][1][8 * t + 2 * qd]);
      auto add = [&](const float4* from, const float4& by) {
        float4 u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = from[k * 32];
#pragma unroll
        for (int k = 0; k < 4; ++k) { acc[k][0] += u[k].x * by.x; acc[k][1] += u[k].y * by.z; acc[k][2] += u[k].z * by.x; acc[k][3] += u[k].w * by.z; }
      };
#pragma unroll 1
      for (int y = early ? last - first : last - first + 1; y > 0; --y, o += Z::kRegion / 16, w += TM) add(o, *w);
      if (early) add(fetched + (x - x0) * 128, *reinterpret_cast<const float4*>(&s_ml[last][0][8 * t + 2 * qd]));
      if (c.open) {
        float4* to = reinterpret_cast<float4*>(record(c)) + part * 128 + lane;
#pragma unroll
        for (int k = 0; k < 4; ++k) __stcg(to + k * 32, make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]));
      } else {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int row = c.seg.row0 + 8 * t + 2 * qd + y;
          if (row >= nrows) continue;
          const int i = verify_row(row), j = row - i * a.G;
          uint32_t* to = reinterpret_cast<uint32_t*>(a.out + (size_t(c.seg.b) * a.Rs + i) * a.ldo + size_t(c.seg.hk * a.G + j) * DH + CPG * g + 2 * f);
#pragma unroll
          for (int k = 0; k < 4; ++k) to[k] = pack_bf16(acc[k][y], acc[k][2 + y]);
        }
      }
    }
  }
  // the unit that goes on behind this CTA
  if (tid == 0 && cuts > 0 && s_cut[cuts - 1].open && !s_cut[cuts - 1].begun) {
    const Segment& seg = s_cut[cuts - 1].seg;
    a.joins[blockIdx.x] = Join{seg.b, seg.hk, seg.row0, s_nr[seg.b] * a.G, (seg.start + seg.blocks - 1) / per_cta + 1};
  }
}

// The units that several CTAs have pieces of: a block a CTA that has a unit's first piece, and eight rows; a warp 16 features.  In a kernel of
// its own, with a unit's slices over many SMs: the last of its CTAs to arrive, joining alone, took 25 us of 90 where eight units of 40 rows
// were in 19 pieces each, and still 2 to 5 where they were in 2 or 3; this one takes 2.
template <int DH, int NT>
__global__ void __launch_bounds__(DH * 2)
attn_int4_join_kernel(const AttnArgs a) {
  using Z = Sizes<DH, NT>;
  constexpr int MT = DH / 16, kBatch = 12;
  extern __shared__ __align__(128) uint8_t smem[];
  float2* const weight = reinterpret_cast<float2*>(smem);      // [pieces][rows] (m, sum), then (weight, -)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3, t = blockIdx.y;
  next_may_launch();
  wait_for_earlier();
  const Join x = a.joins[blockIdx.x];
  if (x.count == 0 || x.row0 + 8 * t >= x.rows) return;
  // the first CTA's second record, then the others' first ones
  auto record = [&](int r) { return a.records + (2 * size_t(blockIdx.x + r) + (r == 0 ? 1 : 0)) * Z::kRecord; };
  float4 v[kBatch];
  auto fetch = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (r0 + u < x.count) v[u] = __ldcg(reinterpret_cast<const float4*>(record(r0 + u)) + (t * MT + warp) * 32 + lane);
  };
  fetch(0);
#pragma unroll 1
  for (int row = warp; row < 8; row += MT) {
    float top = -INFINITY, sum = 0.f;
    for (int r = lane; r < x.count; r += 32) {
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(record(r) + Z::kOBytes / 4) + 8 * t + row);
      weight[r * 8 + row] = ml;
      top = fmaxf(top, ml.x);
    }
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    for (int r = lane; r < x.count; r += 32) sum += weight[r * 8 + row].y * ex2(weight[r * 8 + row].x - top);
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const float inv = 1.f / sum;      // (a row sees itself: its sum is not zero)
    for (int r = lane; r < x.count; r += 32) weight[r * 8 + row].x = ex2(weight[r * 8 + row].x - top) * inv;
  }
  __syncthreads();
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int r0 = 0; r0 < x.count; r0 += kBatch) {
    if (r0) fetch(r0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (r0 + u >= x.count) break;
      const float4 w = *reinterpret_cast<const float4*>(&weight[(r0 + u) * 8 + 2 * qd]);
      acc[0] += v[u].x * w.x; acc[1] += v[u].y * w.z; acc[2] += v[u].z * w.x; acc[3] += v[u].w * w.z;
    }
  }
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int row = x.row0 + 8 * t + 2 * qd + y;
    if (row >= x.rows) continue;
    const int i = a.G == 1 ? row : int(__umulhi(unsigned(row), a.group_inv)), j = row - i * a.G;
    *reinterpret_cast<uint32_t*>(a.out + (size_t(x.b) * a.Rs + i) * a.ldo + size_t(x.hk * a.G + j) * DH + MT * 2 * g + 2 * warp) = pack_bf16(acc[y], acc[2 + y]);
  }
}

// Tiles of the rows that share a kv head: as few as hold 40 rows at most, then as small as that leaves them.
int row_tiles(int rows) {
  const int tiles = ceil_div(rows, 8 * kMostTiles);
  return ceil_div(ceil_div(rows, tiles), 8);
}

laser_status launch_attention(const laser_kv* kv, int n_heads, AttnArgs a, cudaStream_t stream) {
  a.max_seqs = kv->max_seqs;
  a.capacity = int(std::min<int64_t>(kv->capacity_tokens(), INT32_MAX));
  a.Hkv = kv->n_kv_heads; a.G = n_heads / kv->n_kv_heads;
  a.page_table = kv->page_table; a.pages_per_seq = kv->pages_per_seq;
  a.scale = float(1.4426950408889634 / std::sqrt(double(kv->head_dim)));
  a.group_inv = unsigned(((uint64_t(1) << 32) + a.G - 1) / a.G);
  a.part = kv->attn_part;
  const int64_t rows = int64_t(a.Rs) * a.G;
  const int nt = row_tiles(int(std::min<int64_t>(rows, 1 << 28)));
  const int64_t units = a.Hkv * ceil_div(rows, int64_t(8 * nt));          // of a sequence, at most
  // (a sequence's blocks, and a CTA's share of them all, are counted in 32 bits)
  if (units * kv->pages_per_seq > INT32_MAX || units * kv->pages_per_seq * a.B / kv->attn_ctas >= INT32_MAX) {
    set_error("%lld row tiles a sequence (of %d) over caches of %d pages are too many for one call", (long long)units, a.B, kv->pages_per_seq);
    return LASER_ERR_CAPACITY;
  }
  a.vec_out = (reinterpret_cast<uintptr_t>(a.out) | uintptr_t(a.ldo * 2)) % 16 == 0;
  auto launch = [&](auto dh, auto tiles) -> laser_status {
    constexpr int DH = decltype(dh)::value, NT = decltype(tiles)::value;
    using Z = Sizes<DH, NT>;
    const unsigned grid = unsigned(std::min<int64_t>(kv->attn_ctas, units * a.B * kv->pages_per_seq));
    a.records = a.part + size_t(grid) * Z::kPart;
    a.joins = reinterpret_cast<Join*>(a.records + size_t(grid) * 2 * Z::kRecord);
    LASER_CUDA((allow_shared_memory<attn_int4_kernel<DH, NT>>(Z::smem(kMaxSeqs))));
    LASER_CUDA(launch_overlapped(attn_int4_kernel<DH, NT>, dim3(grid), Z::kWarps * 32, size_t(Z::smem(a.B)), stream, a));
    count_launch();
    if (grid > 1) {
      LASER_CUDA(launch_overlapped(attn_int4_join_kernel<DH, NT>, dim3(grid, NT), DH * 2, size_t(grid) * 64, stream, a));
      count_launch();
    }
    return LASER_OK;
  };
  auto by_tiles = [&](auto dh) -> laser_status {
    switch (nt) {
      case 1: return launch(dh, std::integral_constant<int, 1>{});
      case 2: return launch(dh, std::integral_constant<int, 2>{});
      case 3: return launch(dh, std::integral_constant<int, 3>{});
      case 4: return launch(dh, std::integral_constant<int, 4>{});
      default: return launch(dh, std::integral_constant<int, 5>{});
    }
  };
  LASER_TRY(kv->head_dim == 128 ? by_tiles(std::integral_constant<int, 128>{}) : by_tiles(std::integral_constant<int, 64>{}));
  return LASER_OK;
}

}  // namespace

int attention_int4_max_groups() { return kMaxSeqs; }
size_t attention_int4_part_floats(int head_dim, int ctas) {
  auto most = [&](auto... z) { return std::max({decltype(z)::part_floats(ctas)...}); };
  return head_dim == 128 ? most(Sizes<128, 1>{}, Sizes<128, 2>{}, Sizes<128, 3>{}, Sizes<128, 4>{}, Sizes<128, 5>{})
                         : most(Sizes<64, 1>{}, Sizes<64, 2>{}, Sizes<64, 3>{}, Sizes<64, 4>{}, Sizes<64, 5>{});
}

laser_status attention_int4_launch(laser_model* m, laser_kv* kv, int layer, const int32_t* seq_ids, const int32_t* parents, int B, int Rs,
                                   cudaStream_t stream) {
  AttnArgs a{};
  a.seq_ids = seq_ids; a.row_ctx = m->row_ctx; a.row_n = m->row_n; a.parents = parents;
  a.B = B; a.Rs = Rs;
  a.pages = kv->pages4 + size_t(layer) * kv->layer_bytes4();
  a.q = m->q; a.out = m->attn;
  a.ldq = a.ldo = m->dq;         // (the model's heads: another of the same cache shape may have made the cache)
  a.status = m->status;
  return launch_attention(kv, m->cfg.n_heads, a, stream);
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
  return launch_attention(kv, kv->n_heads, a, as_stream(stream));
}
