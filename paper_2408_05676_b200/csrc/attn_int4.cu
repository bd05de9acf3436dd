// Attention of a step's rows over a 4-bit paged cache (int4.cuh): o = sum_t p_t v_t / sum_t p_t, p_t = exp(q . k_t / sqrt(dh)), where row i
// sees the sequence's cached tokens and, of the step's own rows, 0 .. i (chain) or its ancestors and itself (token tree).
//
// The rows of a sequence that share a kv head (rows x n_heads / n_kv_heads) form tiles of 8 NT rows, NT = 1 .. 5.  (sequence, kv head, tile)
// is a unit, of one CTA of four warps or of several ("splits").  A team is a warp, or two where NT > 1.  It walks its pages alone: a page's K
// and V of a head, codes and scales, come by 16-byte copies into the warp's own ring of shared-memory stages (a bulk copy and its barrier cost
// a warp 300 clocks a page, these 100), and the codes become bf16 pairs in registers in the order of the MMA's fragments.  S^T = K Q^T and
// O^T += V^T P^T: tokens and features are the 16-row operand, so that what was unpacked serves all of the tile's rows, eight at a time, and
// few rows waste little.  The sum of P is the product with ones.  Of a team's two warps each takes one page of two, then both pages' P and half
// of the features: half the registers of O a lane, and no page is unpacked twice (one text of 64 thousand tokens, 36 rows: 56 us instead of 66).
//
// A row's bits do not depend on its place in a call: which pages a team sums follows from their numbers and the call's shape (sequences, rows,
// heads, the cache's pages a sequence), a row's softmax references follow from its own scores, and pieces are joined in the order of the teams
// and of the splits.  So neither the other sequences matter, their lengths and rows, nor a row's place among drafts, and strict decoding equals
// greedy decoding here, too.  All pages divided evenly over the SMs, whatever the lengths, with units cut anywhere, gave row results that
// changed in the last bit with the neighbours; it was faster for ragged batches of long texts (one row over 64 texts of 4096 to 8192 tokens 100 us
// instead of 110: a launch ends with CTAs of unequal length here) and for trees of 17 rows (121 instead of 129), and slower for few pages and
// for prompts (one row of 4 heads over 100 tokens 8.7 instead of 3.1; 32 rows of 32 prompts of up to 500 tokens, 32 heads, 53 instead of 42).
//
// What bounds it: the instructions.  A warp-level MMA of 16 x 8 x 16 keeps a scheduler from issuing for eight clocks; a page is 16 NT of
// them, and some 350 other instructions, 200 of them to unpack 4096 codes.  On tensor memory, whose MMAs issue once for 128 tokens, the
// hand-overs between unpacking, products and softmax took longer than what they saved (17 rows: 205 us instead of 122; 36 rows: 69 instead of 52).
//
// The softmax's reference m is a whole number in the exponent of two: raising it multiplies p and O by powers of two, exactly.  It is raised
// only when a score exceeds it by more than 6, which a vote finds; p stays below 2^7, and bf16's and fp32's range is left to what is far below.
//
// Times (us; floors by bytes at 6.56 TB/s in brackets): 32 heads of 128, 9 rows over one text of 512 tokens 7.8 (0.4), over 16 of 256 to 768
// 20.4 (6.7); 40 heads, trees of 17 rows over 64 texts of 256 to 1024 129 (42); 32 heads of 8 kv heads, one row over 64 texts of 4096 to 8192
// 110 (77), 9 rows over one of 65536 52 (13).
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
constexpr int kMaxSeqs = 1024;     // sequences (or prompt chunks) of a call
constexpr int kMostTiles = 5;      // of eight rows in a tile: O takes 80 registers then (of three at most, 36 rows' pages are unpacked twice: 71 us instead of 69)

constexpr int kWarps = 4;          // of a CTA
constexpr int kRun = 2;            // blocks of a team in a run
constexpr int kMostSplits = 256;   // CTAs that share a unit's pages
constexpr int kLarge = 3;          // runs of a large one to a small one's
constexpr int kMostWaves = 4;      // CTAs of a launch that splits pages, in what is resident

// a unit that several CTAs have pieces of (count = 0: none)
struct Join { int b, hk, row0, rows, count; };

template <int DH, int NT>
struct Sizes {
  // A team is a warp, or two that take a page each of every two and half of the features each (one row over long texts: 100 us alone, 112 in
  // twos; 36 rows: 66 alone, 52 in twos)
  static constexpr int kTeam = NT == 1 ? 1 : 2;
  static constexpr int kTeams = kWarps / kTeam;
  static constexpr int kRegsO = NT * DH / 4 / kTeam;     // O registers of a lane
  // CTAs of an SM: as many as the registers allow without spills (one row: five, with 96 registers, 118 us over long texts instead of 115)
  static constexpr int kCtas = NT <= 2 || kRegsO <= 24 ? 4 : kRegsO <= 48 ? 3 : 2;
  static constexpr int kRows = 8 * NT;
  static constexpr int kBlock = q4_block_bytes(DH);      // bytes of a page and head
  static constexpr int kStages = kTeam == 1 ? 4 : 3;     // of a warp's ring (one more: no change)
  static constexpr bool kQInSmem = NT > 1;               // each lane's share of Q is put by and read again for every page
  static constexpr int kQBytes = kQInSmem ? NT * DH / 8 * 4 * 32 : 0;
  static constexpr int kPBytes = kTeam == 1 ? 0 : NT * 2 * 256;          // P of two pages
  static constexpr int kSlices = NT * DH / 16;           // of O: four registers, two neighbouring features of two rows
  static constexpr int kOBytes = kSlices * 512;          // O of a piece
  // A team's memory: its rings, Q and P; when those are done with, O of its piece
  static constexpr int kLoop = kTeam * kStages * kBlock + kQBytes + 2 * kPBytes;
  static constexpr int kRegion = kLoop > kOBytes ? kLoop : kOBytes;
  static constexpr int kSmem = kTeams * kRegion;
  static constexpr int kRecord = kOBytes / 4 + 16 * NT;  // floats of a CTA's piece: O, then (m, sum) of the rows
  static size_t part_floats(int sms) { return size_t(kMostWaves * kCtas) * sms * (kRecord + sizeof(Join) / 4); }
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
  int tiles, splits;                           // of a sequence and kv head: tiles; CTAs that share a tile's pages
  int large, units;                            // those of them that have kLarge times the others' share; (sequence, kv head, tile) altogether
  float* records;                              // their pieces [unit][split]
  Join* joins;                                 // [unit]
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

// -m of rows that have seen nothing: above every score x scale that 32 bits hold (6.1e37), so that the first score a row sees, however low,
// gives it a reference
constexpr float kNothing = 1e38f;

template <int DH, int NT, int CTAS>
__global__ void __launch_bounds__(kWarps * 32, CTAS)
attn_int4_kernel(const AttnArgs a) {
  using Z = Sizes<DH, NT>;
  constexpr int S = Z::kTeam, T = Z::kTeams, ST = Z::kStages, TM = Z::kRows, BLK = Z::kBlock;
  constexpr int KW = DH / 32;            // words of a lane's K (of a token) or V (of two tokens)
  constexpr int VW = KW / S;             // of V, a warp's
  constexpr int CPG = DH / 8;            // output features of a lane
  constexpr int MT = DH / 16;            // 16-feature tiles
  constexpr int OT = MT / S;             // a warp's
  constexpr int QC = DH / 32;            // 16-byte pieces of a lane's share of a Q row
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ unsigned long long s_path[T][64];      // token trees: the rows that a row of the sequence sees
  __shared__ __align__(16) float2 s_ml[T][TM];      // m and sum of the rows of a team's piece
  __shared__ float s_half[S == 1 ? 1 : kWarps][TM];         // what a warp tells the other of its rows: highest scores, or sums
  __shared__ uint32_t s_high[S == 1 ? 1 : kWarps][4 * NT];  // and highest probabilities, of two rows
  __shared__ float s_inv[TM];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3, team = warp / S, half = warp % S;
  // a row is verify row row / G, head row % G of its kv head
  auto verify_row = [&](int row) { return a.G == 1 ? row : int(__umulhi(unsigned(row), a.group_inv)); };

  next_may_launch();
  // ---- the unit, and this CTA's share of its pages ----
  const unsigned split = blockIdx.x / unsigned(a.units), unit = blockIdx.x - split * a.units;
  const unsigned unit_hk = unit / unsigned(a.tiles), tile = unit - unit_hk * a.tiles;
  const int b = int(unit_hk / unsigned(a.Hkv)), hk = int(unit_hk - unsigned(b) * a.Hkv), row0 = int(tile) * TM;
  // Blocks of S pages, in runs of kRun blocks a team, whose teams take the blocks in turn.  Of every `cycle` runs the first splits, the large ones,
  // have kLarge each, the others one.
  constexpr int kRunAll = kRun * T;
  const int large = int(split) < a.large, cycle = a.splits + (kLarge - 1) * a.large;
  const int first_run = large ? int(split) * kLarge : int(split) + (kLarge - 1) * a.large;
  auto block_at = [&](int x) {        // the team's x-th
    const int run = x / kRun, round = large ? run / kLarge : run;
    return (round * cycle + first_run + (large ? run - round * kLarge : 0)) * kRunAll + x % kRun * T + team;
  };
  // (the numbers of the first pages are on their way while the sequence's length is)
  const int32_t* table = a.page_table;
  int ids = -1;
  auto first_pages = [&](int seq) {
    table += size_t(seq) * a.pages_per_seq;
    ids = table[min(block_at(lane) * S + half, a.pages_per_seq - 1)];
  };
  int ctx = 0, nr = 0;
  if (a.row_ctx) {
    // a step's tables were complete before any kernel of the forward began
    ctx = a.row_ctx[b]; nr = a.row_n[b];
    if (nr > 0) first_pages(a.seq_ids[b]);
    wait_for_earlier();
  } else {
    wait_for_earlier();
    const int seq = a.seq_ids[b];
    nr = min(max(a.n_rows[b], 0), a.Rs);
    const bool report = tid == 0 && hk == 0 && tile == 0 && split == 0 && nr > 0;
    if (seq < 0 || seq >= a.max_seqs) {
      if (report) atomicCAS(a.status, 0, LASER_ERR_INVALID_ARG);
      nr = 0;
    } else {
      first_pages(seq);
      ctx = a.seq_len[seq];
      if (ctx < 0 || nr > a.capacity - ctx) {
        if (report) atomicCAS(a.status, 0, LASER_ERR_CAPACITY);
        nr = 0;
      }
    }
  }
  const int nrows = nr * a.G, pages = (ctx + nr + 15) >> 4, blocks = (pages + S - 1) / S;
  const int runs = (blocks + kRunAll - 1) / kRunAll;
  const int parts = nrows <= row0 ? 0 : runs <= kLarge * a.large ? (runs + kLarge - 1) / kLarge : min(a.splits, runs - (kLarge - 1) * a.large);
  if (a.splits > 1 && split == 0 && tid == 0) a.joins[unit] = Join{b, hk, row0, nrows, parts > 1 ? parts : 0};
  if (int(split) >= parts) return;
  auto blocks_of = [&](int w) {        // team w's
    const int whole = blocks / kRunAll, rounds = whole / cycle, ahead = whole - rounds * cycle - first_run, mine = large ? kLarge : 1;
    return kRun * (rounds * mine + min(max(ahead, 0), mine)) + (ahead >= 0 && ahead < mine ? max(blocks - whole * kRunAll - w + T - 1, 0) / T : 0);
  };
  const int n = blocks_of(team);
  if (n > 0) {
    uint8_t* const region = smem + team * Z::kRegion;
    const uint32_t ring_at = smem_u32(region) + half * (ST * BLK) + lane * 16;
    // ---- copies: of 32 blocks each lane holds the number of one's page (none behind the last) ----
    if (S == 2 && block_at(lane) * S + half >= pages) ids = -1;
    auto request = [&](int x, int s) {
      if (x > 0 && (x & 31) == 0) {
        const int page = x + lane < n ? block_at(x + lane) * S + half : pages;
        ids = page < pages ? table[page] : -1;
      }
      const int id = __shfl_sync(0xffffffffu, ids, x & 31);
      if (S == 1 || id >= 0) {
        const uint8_t* src = a.pages + (size_t(id) * a.Hkv + hk) * BLK + lane * 16;
#pragma unroll
        for (int y = 0; y + 512 <= BLK; y += 512) copy16(ring_at + s * BLK + y, src + y);
        if (BLK % 512 && lane < BLK % 512 / 16) copy16(ring_at + s * BLK + BLK / 512 * 512, src + BLK / 512 * 512);
      }
    };
#pragma unroll 1
    for (int s = 0; s < ST; ++s) {
      if (s < n) request(s, s);
      copies_end();
    }

    if (a.parents && half == 0) {
      unsigned long long mask[2];
      tree_paths(a.parents + size_t(b) * a.Rs, nr, lane, mask);
      s_path[team][lane] = mask[0];
      s_path[team][lane + 32] = mask[1];
      __syncwarp();
    }
    // ---- Q: a lane's features are those of its K words ----
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

    int stage = 0;
#pragma unroll 1
    for (int it = 0; it < n; ++it) {
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
      const int blk = block_at(it), page = blk * S + half;        // (the second of a team's may be one too many: all of it is masked)
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
      // (P enters the second product as bf16, in the numerator and in the sum, as in the attention over a bf16 cache: results are off by 0.0023 of
      // their size where their own rounding to bf16 takes 0.0017; what the rounding leaves, as a second operand, would be that many MMAs again)
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
        // Of the rows that have one above 2^6, and of no others: a row's references follow from its own scores.
        uint32_t high[NT];
        float top[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          high[t] = max2(pack_bf16(ex2(exponent(t, 0)), ex2(exponent(t, 1))), pack_bf16(ex2(exponent(t, 2)), ex2(exponent(t, 3))));
#pragma unroll
          for (int y = 0; y < 2; ++y) top[t][y] = fmaxf(x[t][y], x[t][2 + y]);
#pragma unroll
          for (int d = 4; d <= 16; d <<= 1) {
            high[t] = max2(high[t], __shfl_xor_sync(0xffffffffu, high[t], d));
#pragma unroll
            for (int y = 0; y < 2; ++y) top[t][y] = fmaxf(top[t][y], __shfl_xor_sync(0xffffffffu, top[t][y], d));
          }
          if (S == 2 && g == 0) {
            s_high[S == 1 ? 0 : warp][4 * t + qd] = high[t];
            s_half[S == 1 ? 0 : warp][8 * t + 2 * qd] = top[t][0];
            s_half[S == 1 ? 0 : warp][8 * t + 2 * qd + 1] = top[t][1];
          }
        }
        if (S == 2) team_sync(team);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (S == 2) high[t] = max2(high[t], s_high[S == 1 ? 0 : warp ^ 1][4 * t + qd]);
          float down[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            if (S == 2) top[t][y] = fmaxf(top[t][y], s_half[S == 1 ? 0 : warp ^ 1][8 * t + 2 * qd + y]);
            const bool raise = (high[t] >> (16 * y) & 0xffffu) > 0x4280u;
            const float next = raise ? fminf(shift[t][y], -ceilf(__fmul_rn(top[t][y], a.scale))) : shift[t][y];
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
        if (it - 1 + ST < n) request(it - 1 + ST, stage == 0 ? ST - 1 : stage - 1);
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
        if (it + ST < n) request(it + ST, stage);
        copies_end();
      }
      if (++stage == ST) stage = 0;
    }

    // ---- the team's piece ----
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
    copies_done();
    __syncwarp();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (row0 + 8 * t >= nrows) break;      // (no row of the tile)
#pragma unroll
      for (int f = 0; f < OT; ++f)
        reinterpret_cast<float4*>(region)[(t * MT + half * OT + f) * 32 + lane] = make_float4(o[t][f][0], o[t][f][1], o[t][f][2], o[t][f][3]);
      if (half == 0 && g == 0) {
#pragma unroll
        for (int y = 0; y < 2; ++y) s_ml[team][8 * t + 2 * qd + y] = make_float2(shift[t][y] == kNothing ? -INFINITY : -shift[t][y], sums[t][y]);
      }
    }
  }
  __syncthreads();

  // ---- the teams' pieces, weighted and added in the order of the teams; what it comes to is the result, or this CTA's piece of it.  (The
  // division comes last in either case: a row's bits are the same whether or not there are pages behind it that it does not see.) ----
  int teams = 1;
#pragma unroll
  for (int w = 1; w < T; ++w) teams += blocks_of(w) > 0;
  const int live = min(TM, nrows - row0);
  float* const record = a.records + (size_t(unit) * a.splits + split) * Z::kRecord;
  if (tid < live) {
    float2 ml[T];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < T; ++x) {
      ml[x] = x < teams ? s_ml[x][tid] : make_float2(-INFINITY, 0.f);
      m = fmaxf(m, ml[x].x);
    }
    const float zero = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int x = 0; x < T; ++x) {
      const float w = ex2(ml[x].x - zero);
      l += ml[x].y * w;
      if (x < teams) s_ml[x][tid].x = w;
    }
    s_inv[tid] = 1.f / l;                          // (a row sees itself: its sum over all pages is not zero)
    if (parts > 1) __stcg(reinterpret_cast<float2*>(record + Z::kOBytes / 4) + tid, make_float2(m, l));
  }
  __syncthreads();
#pragma unroll 1
  for (int part = warp; part < Z::kSlices / 4; part += kWarps) {      // four slices of eight rows
    const int t = part / (MT / 4), f = part % (MT / 4) * 4;
    if (8 * t >= live) break;
    float acc[4][4] = {};
#pragma unroll
    for (int x = 0; x < T; ++x) {
      if (x >= teams) break;
      const float4* from = reinterpret_cast<const float4*>(smem + x * Z::kRegion) + part * 128 + lane;
      const float4 w = *reinterpret_cast<const float4*>(&s_ml[x][8 * t + 2 * qd]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 u = from[k * 32];
        acc[k][0] += u.x * w.x; acc[k][1] += u.y * w.z; acc[k][2] += u.z * w.x; acc[k][3] += u.w * w.z;
      }
    }
    if (parts > 1) {
      float4* to = reinterpret_cast<float4*>(record) + part * 128 + lane;
#pragma unroll
      for (int k = 0; k < 4; ++k) __stcg(to + k * 32, make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]));
      continue;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int at = 8 * t + 2 * qd + y;
      if (at >= live) continue;
      const int row = row0 + at, i = verify_row(row), j = row - i * a.G;
      const float inv = s_inv[at];
      bf16* dst = a.out + (size_t(b) * a.Rs + i) * a.ldo + size_t(hk * a.G + j) * DH + CPG * g + 2 * f;
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = pack_bf16(acc[k][y] * inv, acc[k][2 + y] * inv);
      if (a.vec_out) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint32_t*>(dst + 2 * k) = w[k];
      }
    }
  }
}

// The units that several CTAs have pieces of: a block a unit and eight rows, a warp 16 features.  In a kernel of its own, with a unit's slices
// over many SMs: the last of its CTAs to arrive, joining alone, took 25 us of 90 where eight units of 40 rows were in 19 pieces each, and
// still 2 to 5 where they were in 2 or 3; this one takes 2.
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
  auto record = [&](int r) { return a.records + (size_t(blockIdx.x) * a.splits + r) * Z::kRecord; };
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

// `part`: room for partial results, which calls that may run at the same time do not share.
laser_status launch_attention(const laser_kv* kv, int n_heads, AttnArgs a, float* part, cudaStream_t stream) {
  a.max_seqs = kv->max_seqs;
  a.capacity = int(std::min<int64_t>(kv->capacity_tokens(), INT32_MAX));
  a.Hkv = kv->n_kv_heads; a.G = n_heads / kv->n_kv_heads;
  a.page_table = kv->page_table; a.pages_per_seq = kv->pages_per_seq;
  a.scale = float(1.4426950408889634 / std::sqrt(double(kv->head_dim)));
  a.group_inv = unsigned(((uint64_t(1) << 32) + a.G - 1) / a.G);
  a.records = part;
  const int64_t rows = int64_t(a.Rs) * a.G;
  const int nt = row_tiles(int(std::min<int64_t>(rows, 1 << 28)));
  const int64_t tiles = ceil_div(rows, int64_t(8 * nt)), units = int64_t(a.B) * a.Hkv * tiles;
  // (a sequence's pages, over all its units, and a launch's CTAs are counted in 32 bits; the share of an SM bounds what one call may take)
  if (a.Hkv * tiles * kv->pages_per_seq > INT32_MAX || units * kv->pages_per_seq / kv->attn_sms >= INT32_MAX || units > INT32_MAX) {
    set_error("%lld row tiles a sequence (of %d) over caches of %d pages are too many for one call", (long long)(a.Hkv * tiles), a.B, kv->pages_per_seq);
    return LASER_ERR_CAPACITY;
  }
  a.tiles = int(tiles);
  a.vec_out = (reinterpret_cast<uintptr_t>(a.out) | uintptr_t(a.ldo * 2)) % 16 == 0;
  auto launch = [&](auto dh, auto tiles_tag) -> laser_status {
    constexpr int DH = decltype(dh)::value, NT = decltype(tiles_tag)::value;
    using Z = Sizes<DH, NT>;
    const int64_t resident = int64_t(kv->attn_sms) * Z::kCtas, runs = ceil_div(ceil_div(kv->pages_per_seq, Z::kTeam), kRun * Z::kTeams);      // (of a text as long as may be)
    // As many CTAs as are resident, or less where that leaves each the same runs at most.  Texts of several sequences may differ in length: then
    // more, as long as each has pages enough, the large ones first and small ones for the end (one row over 64 texts of 4096 to 8192: one CTA a
    // unit 135 us, two 122, four of a size 116, two large and two small 110, eight of a size 118).
    const int64_t wave = resident / units, waves = a.B > 1 ? std::min<int64_t>(kMostWaves * resident / units, kv->pages_per_seq / 32) : 0;
    a.large = 0;
    if (waves > std::max<int64_t>(wave, 1)) {
      a.splits = int(std::min<int64_t>({waves, runs, kMostSplits}));
      a.large = a.splits / 2;
    } else {
      a.splits = int(std::max<int64_t>(1, std::min<int64_t>({wave, runs, kMostSplits})));
      a.splits = ceil_div(int(runs), ceil_div(int(runs), a.splits));
    }
    a.units = int(units);
    a.joins = reinterpret_cast<Join*>(a.records + size_t(units) * a.splits * Z::kRecord);
    // (two tiles: four CTAs an SM take 128 registers a thread, which makes one slower: 16 texts of 256 to 768, 9 rows of 32 heads, 20.8 us instead
    // of 23.2, one text of 512 9.7 instead of 8.3)
    constexpr int kFew = NT == 2 ? 3 : Z::kCtas;
    const dim3 grid(unsigned(units) * a.splits);
    if (NT == 2 && units * a.splits <= kFew * kv->attn_sms) {
      LASER_CUDA((allow_shared_memory<attn_int4_kernel<DH, NT, kFew>>(Z::kSmem)));
      LASER_CUDA(launch_overlapped(attn_int4_kernel<DH, NT, kFew>, grid, kWarps * 32, size_t(Z::kSmem), stream, a));
    } else {
      LASER_CUDA((allow_shared_memory<attn_int4_kernel<DH, NT, Z::kCtas>>(Z::kSmem)));
      LASER_CUDA(launch_overlapped(attn_int4_kernel<DH, NT, Z::kCtas>, grid, kWarps * 32, size_t(Z::kSmem), stream, a));
    }
    count_launch();
    if (a.splits > 1) {
      LASER_CUDA(launch_overlapped(attn_int4_join_kernel<DH, NT>, dim3(unsigned(units), NT), DH * 2, size_t(a.splits) * 64, stream, a));
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
size_t attention_int4_part_floats(int head_dim, int sms) {
  auto most = [&](auto... z) { return std::max({decltype(z)::part_floats(sms)...}); };
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
  return launch_attention(kv, m->cfg.n_heads, a, m->attn4_part, stream);
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
  return launch_attention(kv, kv->n_heads, a, kv->attn_part, as_stream(stream));
}
