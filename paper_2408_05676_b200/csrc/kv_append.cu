// Appending the keys and values of a step's rows to a paged cache (bf16, or the 4-bit form of int4.cuh), rotary embedding of queries and
// keys on the way; and the copies in and out of a 4-bit cache.
//
// Row i of sequence b sits at position len + depth(i) (chain: len + i) and goes to slot len + i.  The pair (x_j, x_{j + dh/2}) turns by
// position x theta^(-2j / dh); angles in 64 bits, since fp32 products are off by 1e-2 rad at position 1e5, the rotation itself in fp32.
// A block takes one row and a share of its heads, so that a row's sines are worked out once per block; a lane holds four features
// (8 or 16 bytes a load), head_dim / 4 lanes a head, the rotation's partner and a group's extremes come by shuffles.  (Eight features a lane, with
// no shuffle for the rotation, took twice the code and 80 registers: 128 us instead of 72 for the prompts below.)
//
// Times into a 4-bit cache (us; floors by bytes at 6.56 TB/s in brackets): one row of 4 heads of 64 4.3, 16 x 9 rows of 32 heads of 128 7.1 (0.7), both
// two dependent trips to memory and the sines; 64 trees of 17 rows of 40 heads in fp32 16.5 (8.7); prompts of 10 thousand rows of 32 heads, 8 kv heads,
// 62 (32): bound by instructions, of which codes of keys and values take half (queries alone: 33 us).
#include <algorithm>
#include <type_traits>

#include "int4.cuh"
#include "model.cuh"

namespace laser {
namespace {

using bf16 = __nv_bfloat16;
constexpr int kAppendThreads = 256;
constexpr int kRowsMost = 8;      // rows of a block

struct AppendArgs {
  // rows: from a step's tables (row_pos: slot, -1 = none; rope), or from the sequences' lengths, or a run of one sequence (run_seq >= 0)
  const int32_t *row_pos, *row_seq;
  const float* rope;
  const int32_t *seq_ids, *n_rows, *parents, *seq_len;
  const double* inv_freq;
  int32_t* status;
  int run_seq, run_pos, Rs, max_seqs, capacity;
  long long total;              // rows
  int per_block;                // of them a block's
  int H, Hkv;
  const void *q, *k, *v;
  long long ldq, ldk, ldv;      // elements between rows
  int vec;                      // four features may be loaded at once
  bf16 *q_out, *k_out, *v_out;
  const int32_t* page_table;
  int pages_per_seq;
  bf16* pages;                  // one of the two: this layer's pages
  uint8_t* pages4;
};

// Four features of a lane as they came, fetched before they are needed.
template <typename T> struct Raw { T x[4]; };
template <typename T>
__device__ __forceinline__ Raw<T> fetch4(const T* p, int vec) {
  Raw<T> r;
  if (vec) {
    if (sizeof(T) == 2) *reinterpret_cast<uint2*>(&r) = *reinterpret_cast<const uint2*>(p);
    else *reinterpret_cast<uint4*>(&r) = *reinterpret_cast<const uint4*>(p);
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) r.x[u] = p[u];
  }
  return r;
}

__device__ __forceinline__ uint32_t two_bf16(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <typename T, int DH>
__global__ void __launch_bounds__(kAppendThreads)
kv_append_kernel(const AppendArgs a) {
  constexpr int LPH = DH / 4, HPW = 32 / LPH;       // lanes of a head, heads of a warp
  constexpr int W = kAppendThreads / 32;
  __shared__ float2 s_cs[kRowsMost][DH / 2];
  __shared__ int s_pos[kRowsMost];                  // a row's position
  __shared__ void* s_dst[kRowsMost];          // its page (null: the row is not one)
  __shared__ int s_slot[kRowsMost];                 // its place in the page
  next_may_launch();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, l = lane % LPH;
  const long long row0 = (long long)blockIdx.x * a.per_block;
  const int here = int(min((long long)a.per_block, a.total - row0));
  wait_for_earlier();

  // ---- the rows: a thread each ----
  if (tid < here) {
    const long long r = row0 + tid;
    int slot = -1, seq = 0, pos = 0;
    if (a.row_pos) {
      slot = a.row_pos[r]; seq = a.row_seq[r];
    } else if (a.run_seq >= 0) {
      seq = a.run_seq; slot = a.run_pos + int(r);
    } else {
      const int b = int(r / a.Rs), i = int(r - (long long)b * a.Rs);
      seq = a.seq_ids[b];
      const int nr = min(max(a.n_rows[b], 0), a.Rs);
      if (i < nr) {
        if (seq < 0 || seq >= a.max_seqs) {
          atomicCAS(a.status, 0, LASER_ERR_INVALID_ARG);
        } else {
          const int ctx = a.seq_len[seq];
          if (ctx < 0 || nr > a.capacity - ctx) {
            atomicCAS(a.status, 0, LASER_ERR_CAPACITY);
          } else {
            slot = pos = ctx + i;
            if (a.parents) {
              int depth = 0;
              for (int j = i; j > 0; ++depth) {     // parents are earlier rows: at most i steps
                const int pj = a.parents[size_t(b) * a.Rs + j];
                if (pj < 0 || pj >= j) { atomicCAS(a.status, 0, LASER_ERR_INVALID_ARG); break; }
                j = pj;
              }
              pos = ctx + depth;
            }
          }
        }
      }
    }
    s_pos[tid] = pos;
    s_slot[tid] = slot & 15;
    void* dst = nullptr;
    if (slot >= 0) {
      const size_t page = size_t(a.page_table[size_t(seq) * a.pages_per_seq + (slot >> 4)]);
      dst = a.pages4 ? static_cast<void*>(a.pages4 + page * a.Hkv * q4_block_bytes(DH)) : static_cast<void*>(a.pages + page * 2 * a.Hkv * 16 * DH);
    }
    s_dst[tid] = dst;
  }
  __syncthreads();
  // ---- their angles ----
  if (a.run_seq < 0) {
    for (int x = tid; x < here * (DH / 2); x += kAppendThreads) {
      const int rr = x / (DH / 2), j = x % (DH / 2);
      if (!s_dst[rr]) continue;
      if (a.row_pos) {
        s_cs[rr][j] = *reinterpret_cast<const float2*>(a.rope + (size_t(row0 + rr) * (DH / 2) + j) * 2);
      } else {
        double s, c;
        sincos(double(s_pos[rr]) * a.inv_freq[j], &s, &c);
        s_cs[rr][j] = make_float2(float(c), float(s));
      }
    }
    __syncthreads();
  }

  // ---- a warp takes a share of one row's heads, one (or two of 64) at a time, kAhead of them on their way together ----
  const int warps_of_row = W / a.per_block, rr = warp / warps_of_row;
  if (rr >= here || !s_dst[rr]) return;
  const int part = blockIdx.y * warps_of_row + warp % warps_of_row, parts = gridDim.y * warps_of_row;
  const long long r = row0 + rr;
  const int t = s_slot[rr];
  uint8_t* const page = static_cast<uint8_t*>(s_dst[rr]);
  float cs[4], sn[4];        // the lane's sines, with the sign that its half of the head takes them with
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float2 x = s_cs[rr][(4 * l + u) & (DH / 2 - 1)];
    cs[u] = x.x;
    sn[u] = l < LPH / 2 ? -x.y : x.y;
  }
  constexpr int kAhead = 4;
  auto heads = [&](auto kind_tag, const T* src, int count, bf16* to) {
    constexpr int kKind = decltype(kind_tag)::value;       // 0 = q, 1 = k, 2 = v
    const int hl = lane / LPH;
    for (int h0 = part * HPW; h0 < count; h0 += kAhead * parts * HPW) {
      Raw<T> raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int h = h0 + u * parts * HPW + hl;
        raw[u] = h < count ? fetch4(src + h * DH + 4 * l, a.vec) : Raw<T>{};
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (h0 + u * parts * HPW >= count) break;
        const int h = h0 + u * parts * HPW + hl;
        const bool live = h < count;
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = float(raw[u].x[c]);
        if (kKind != 2 && a.run_seq < 0) {
          float p[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) p[c] = __shfl_xor_sync(0xffffffffu, y[c], LPH / 2);
#pragma unroll
          for (int c = 0; c < 4; ++c) y[c] = __fadd_rn(__fmul_rn(y[c], cs[c]), __fmul_rn(p[c], sn[c]));
        }
        uint2 held;
        if (kKind == 0 || !a.pages4) {
          held = make_uint2(two_bf16(y[0], y[1]), two_bf16(y[2], y[3]));
          if (kKind > 0 && live)
            *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(page) + (size_t(kKind - 1) * a.Hkv + h) * 16 * DH + t * DH + 4 * l) = held;
        } else {
          q4_finite(y);
          const Q4Scale sc = q4_scale(y);
          float at[4];
          q4_codes(y, sc, at);
          uint8_t* blk = page + h * q4_block_bytes(DH);
          if (kKind == 1) {
            uint32_t kw = __byte_perm(q4_two(at[0], at[2]), q4_two(at[1], at[3]), 0x5410) << 3;      // codes at bits 3, 19, 7, 23
            if (l & 1) kw = __funnelshift_l(kw, kw, 8);
            kw |= __shfl_xor_sync(0xffffffffu, kw, 1);
            if (live && !(l & 1)) *reinterpret_cast<uint32_t*>(blk + q4_k_codes(DH, t, l >> 1)) = kw;
            if (live && !(l & 7)) *reinterpret_cast<uint32_t*>(blk + q4_k_scale(DH, t, l >> 3)) = sc.s | sc.z << 16;
          } else if (live) {
            *reinterpret_cast<uint16_t*>(blk + q4_v_codes(DH, t, l)) = uint16_t(__byte_perm(q4_two(at[0], at[1]), q4_two(at[2], at[3]), 0x0040));
            if (!(l & 7)) {
              uint8_t* p = blk + q4_v_scale(DH, t, l >> 3);
              *reinterpret_cast<uint16_t*>(p) = uint16_t(sc.s);
              *reinterpret_cast<uint16_t*>(p + 4) = uint16_t(sc.z);
            }
          }
          if (to) held = make_uint2(q4_held2(at[0], at[1], sc), q4_held2(at[2], at[3], sc));
        }
        if (to && live) *reinterpret_cast<uint2*>(to + (size_t(r) * count + h) * DH + 4 * l) = held;
      }
    }
  };
  heads(std::integral_constant<int, 1>{}, static_cast<const T*>(a.k) + r * a.ldk, a.Hkv, a.k_out);
  heads(std::integral_constant<int, 2>{}, static_cast<const T*>(a.v) + r * a.ldv, a.Hkv, a.v_out);
  if (a.H) heads(std::integral_constant<int, 0>{}, static_cast<const T*>(a.q) + r * a.ldq, a.H, a.q_out);
}

// What a 4-bit cache holds of tokens [pos0, pos0 + n) of one sequence, as bf16: a thread takes four features of K or V.
__global__ void export_q4_kernel(const uint8_t* __restrict__ pages, const int32_t* __restrict__ pt, int Hkv, int dh, int pos0, int n,
                                 int vec, bf16* __restrict__ k, bf16* __restrict__ v) {
  const int c4s = dh / 4;
  const size_t total = size_t(n) * 2 * Hkv * c4s;
  for (size_t idx = size_t(blockIdx.x) * blockDim.x + threadIdx.x; idx < total; idx += size_t(gridDim.x) * blockDim.x) {
    const int c4 = int(idx % c4s), h = int(idx / c4s % Hkv), is_v = int(idx / (size_t(c4s) * Hkv) % 2);
    const size_t tok = idx / (size_t(c4s) * Hkv * 2);
    const int slot = pos0 + int(tok), t = slot & 15;
    const uint8_t* blk = pages + (size_t(pt[slot >> 4]) * Hkv + h) * q4_block_bytes(dh);
    Q4Scale sc;
    uint32_t codes;
    if (is_v) {
      const uint8_t* p = blk + q4_v_scale(dh, t, c4 >> 3);
      sc.s = *reinterpret_cast<const uint16_t*>(p);
      sc.z = *reinterpret_cast<const uint16_t*>(p + 4);
      codes = *reinterpret_cast<const uint16_t*>(blk + q4_v_codes(dh, t, c4));
    } else {
      const uint32_t sz = *reinterpret_cast<const uint32_t*>(blk + q4_k_scale(dh, t, c4 >> 3));
      sc.s = sz & 0xffffu; sc.z = sz >> 16;
      uint32_t w = *reinterpret_cast<const uint32_t*>(blk + q4_k_codes(dh, t, c4 >> 1));
      w = __funnelshift_r(w, w, 3 + 8 * (c4 & 1));           // features at bits 0, 16, 4, 20
      codes = (w & 15u) | (w >> 16 & 15u) << 4 | (w >> 4 & 15u) << 8 | (w >> 20 & 15u) << 12;
    }
    float at[4];
    for (int u = 0; u < 4; ++u) at[u] = float(16 + int(codes >> (4 * u) & 15u));
    const uint2 held = make_uint2(q4_held2(at[0], at[1], sc), q4_held2(at[2], at[3], sc));
    bf16* to = (is_v ? v : k) + (tok * Hkv + h) * dh + 4 * c4;
    if (vec) *reinterpret_cast<uint2*>(to) = held;
    else for (int u = 0; u < 4; ++u) to[u] = reinterpret_cast<const bf16*>(&held)[u];
  }
}

// compact_path_kernel for a 4-bit cache (ascending moves; a thread owns the same pieces of every token that it moves).
__global__ void compact_path_q4_kernel(uint8_t* __restrict__ pages, size_t layer_bytes, const int32_t* __restrict__ page_table, int pages_per_seq,
                                       int Hkv, int dh, const int32_t* seq_ids, const int32_t* seq_len, const int32_t* path_rows,
                                       const int32_t* n_accept, int row_stride, int max_seqs, int capacity) {
  next_may_launch();
  wait_for_earlier();
  const int b = blockIdx.x, layer = blockIdx.y;
  const int seq = seq_ids[b];
  if (seq < 0 || seq >= max_seqs) return;
  const int a = min(n_accept[b], row_stride - 1), ctx = seq_len[seq];
  const int32_t* pt = page_table + size_t(seq) * pages_per_seq;
  uint8_t* base = pages + size_t(layer) * layer_bytes;
  const int kw = dh / 8, ks = dh / 32, vw = dh / 4, vs = dh / 32, per_head = kw + ks + vw + vs;
  for (int c = threadIdx.x; c < Hkv * per_head; c += blockDim.x) {
    const int h = c / per_head, x = c % per_head;
    for (int j = 0; j < a; ++j) {
      const int row = path_rows[size_t(b) * row_stride + j];
      const int src = ctx + row, dst = ctx + j + 1;
      if (row < j + 1 || src >= capacity || src == dst) continue;
      const uint8_t* s = base + (size_t(pt[src >> 4]) * Hkv + h) * q4_block_bytes(dh);
      uint8_t* d = base + (size_t(pt[dst >> 4]) * Hkv + h) * q4_block_bytes(dh);
      const int ts = src & 15, td = dst & 15;
      if (x < kw) {
        *reinterpret_cast<uint32_t*>(d + q4_k_codes(dh, td, x)) = *reinterpret_cast<const uint32_t*>(s + q4_k_codes(dh, ts, x));
      } else if (x < kw + ks) {
        *reinterpret_cast<uint32_t*>(d + q4_k_scale(dh, td, x - kw)) = *reinterpret_cast<const uint32_t*>(s + q4_k_scale(dh, ts, x - kw));
      } else if (x < kw + ks + vw) {
        *reinterpret_cast<uint16_t*>(d + q4_v_codes(dh, td, x - kw - ks)) = *reinterpret_cast<const uint16_t*>(s + q4_v_codes(dh, ts, x - kw - ks));
      } else {
        const int to = q4_v_scale(dh, td, x - kw - ks - vw), from = q4_v_scale(dh, ts, x - kw - ks - vw);
        *reinterpret_cast<uint16_t*>(d + to) = *reinterpret_cast<const uint16_t*>(s + from);
        *reinterpret_cast<uint16_t*>(d + to + 4) = *reinterpret_cast<const uint16_t*>(s + from + 4);
      }
    }
  }
}

laser_status launch_append(AppendArgs a, int64_t rows, int dh, int dtype, cudaStream_t stream) {
  // a row a warp where rows are many; where they are few, up to eight warps a row and several blocks
  const int heads = std::max(a.H, a.Hkv), items = ceil_div(heads, 128 / dh), warps = kAppendThreads / 32;
  a.total = rows;
  a.per_block = rows >= 592 * 8 ? 8 : rows >= 592 * 4 ? 4 : rows >= 592 * 2 ? 2 : 1;
  const int64_t blocks = ceil_div(rows, int64_t(a.per_block));
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(ceil_div(items * a.per_block, warps), 592 / blocks)));
  auto launch = [&](auto kernel) -> laser_status {
    LASER_CUDA(launch_overlapped(kernel, dim3(unsigned(blocks), unsigned(parts)), kAppendThreads, 0, stream, a));
    return LASER_OK;
  };
  if (dtype == LASER_DTYPE_F32) LASER_TRY(dh == 128 ? launch(kv_append_kernel<float, 128>) : launch(kv_append_kernel<float, 64>));
  else LASER_TRY(dh == 128 ? launch(kv_append_kernel<bf16, 128>) : launch(kv_append_kernel<bf16, 64>));
  count_launch();
  return LASER_OK;
}

AppendArgs append_args(const laser_kv* kv, int layer) {
  AppendArgs a{};
  a.run_seq = -1;
  a.Hkv = kv->n_kv_heads; a.max_seqs = kv->max_seqs;
  a.capacity = int(std::min<int64_t>(kv->capacity_tokens(), INT32_MAX));
  a.seq_len = kv->seq_len; a.inv_freq = kv->inv_freq; a.status = kv->status;
  a.page_table = kv->page_table; a.pages_per_seq = kv->pages_per_seq;
  if (kv->pages4) a.pages4 = kv->pages4 + size_t(layer) * kv->layer_bytes4();
  else a.pages = kv->pages + size_t(layer) * kv->layer_elems();
  return a;
}

// whether four features may be loaded at once
bool four_at_once(const void* p, int64_t ld, int size) { return (reinterpret_cast<uintptr_t>(p) | uintptr_t(ld * size)) % (4 * size) == 0; }

}  // namespace

// Keys, values and queries of a step whose rows a model's tables describe: fp32 [rows, (H + 2 Hkv) head_dim].
laser_status append_step_rows(laser_model* m, laser_kv* kv, int layer, const float* qkv, int64_t ld, bool queries, int rows, cudaStream_t stream) {
  AppendArgs a = append_args(kv, layer);
  a.row_pos = m->row_pos; a.row_seq = m->row_seq; a.rope = m->rope;
  a.H = queries ? m->cfg.n_heads : 0;
  a.q = qkv; a.k = qkv + size_t(a.H) * m->cfg.head_dim; a.v = qkv + size_t(a.H + a.Hkv) * m->cfg.head_dim;
  a.ldq = a.ldk = a.ldv = ld;
  a.vec = 1;
  a.q_out = m->q;
  return launch_append(a, rows, m->cfg.head_dim, LASER_DTYPE_F32, stream);
}

laser_status kv_copy_q4(const laser_kv* kv, int seq, int layer, int pos0, int n, void* k, void* v, bool to_pages, cudaStream_t stream) {
  if (to_pages) {
    AppendArgs a = append_args(kv, layer);
    a.run_seq = seq; a.run_pos = pos0;
    a.k = k; a.v = v;
    a.ldk = a.ldv = int64_t(kv->n_kv_heads) * kv->head_dim;
    a.vec = four_at_once(k, 0, 2) && four_at_once(v, 0, 2);
    return launch_append(a, n, kv->head_dim, LASER_DTYPE_BF16, stream);
  }
  const int vec = four_at_once(k, 0, 2) && four_at_once(v, 0, 2);
  const size_t total = size_t(n) * 2 * kv->n_kv_heads * (kv->head_dim / 4);
  export_q4_kernel<<<unsigned(std::min<size_t>(ceil_div<size_t>(total, 256), 4096)), 256, 0, stream>>>(
      kv->pages4 + size_t(layer) * kv->layer_bytes4(), kv->page_table + size_t(seq) * kv->pages_per_seq, kv->n_kv_heads, kv->head_dim, pos0, n,
      vec, static_cast<bf16*>(k), static_cast<bf16*>(v));
  count_launch();
  LASER_CUDA(cudaGetLastError());
  return LASER_OK;
}

laser_status compact_path_q4(laser_kv* kv, const int32_t* seq_ids, const int32_t* path_rows, const int32_t* n_accept, int B, int row_stride,
                             cudaStream_t stream) {
  LASER_CUDA(launch_overlapped(compact_path_q4_kernel, dim3(unsigned(B), unsigned(kv->n_layers)), 256, 0, stream, kv->pages4, kv->layer_bytes4(),
                               kv->page_table, kv->pages_per_seq, kv->n_kv_heads, kv->head_dim, seq_ids, kv->seq_len, path_rows, n_accept, row_stride,
                               kv->max_seqs, int(std::min<int64_t>(kv->capacity_tokens(), INT32_MAX))));
  count_launch();
  return LASER_OK;
}

}  // namespace laser

using namespace laser;

LASER_API laser_status laser_kv_append(laser_kv* kv, int32_t layer, const int32_t* seq_ids, const int32_t* parents, const int32_t* n_rows,
                                       int32_t B, int32_t rows, int32_t dtype, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                       const void* v, int64_t v_stride, void* q_out, void* k_out, void* v_out, void* stream) {
  LASER_REQUIRE(kv && seq_ids && n_rows && k && v, "null argument");
  LASER_REQUIRE((q != nullptr) == (q_out != nullptr), "q and q_out go together");
  LASER_REQUIRE(layer >= 0 && layer < kv->n_layers, "layer %d out of range", layer);
  LASER_REQUIRE(B >= 0 && rows >= 1 && int64_t(B) * rows <= INT32_MAX, "B = %d sequences of %d rows", B, rows);
  LASER_REQUIRE(!parents || rows <= 64, "a token tree has at most 64 rows (rows = %d)", rows);
  LASER_REQUIRE(dtype == LASER_DTYPE_BF16 || dtype == LASER_DTYPE_F32, "dtype = %d", dtype);
  if (kv->head_dim != 64 && kv->head_dim != 128) { set_error("head_dim = %d (must be 64 or 128)", kv->head_dim); return LASER_ERR_UNSUPPORTED; }
  const int64_t wq = int64_t(kv->n_heads) * kv->head_dim, wk = int64_t(kv->n_kv_heads) * kv->head_dim;
  LASER_REQUIRE((!q || q_stride >= wq) && k_stride >= wk && v_stride >= wk, "rows overlap: strides %lld, %lld, %lld", (long long)q_stride,
                (long long)k_stride, (long long)v_stride);
  const int size = dtype == LASER_DTYPE_BF16 ? 2 : 4;
  LASER_REQUIRE((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % size == 0, "q, k, v must be aligned to their type");
  LASER_REQUIRE(((reinterpret_cast<uintptr_t>(q_out) | reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 7) == 0,
                "q_out, k_out and v_out must be 8-byte aligned");
  if (B == 0) return LASER_OK;
  AppendArgs a = append_args(kv, layer);
  a.seq_ids = seq_ids; a.n_rows = n_rows; a.parents = parents; a.Rs = rows;
  a.H = q ? kv->n_heads : 0;
  a.q = q; a.k = k; a.v = v;
  a.ldq = q_stride; a.ldk = k_stride; a.ldv = v_stride;
  a.vec = (!q || four_at_once(q, q_stride, size)) && four_at_once(k, k_stride, size) && four_at_once(v, v_stride, size);
  a.q_out = static_cast<bf16*>(q_out); a.k_out = static_cast<bf16*>(k_out); a.v_out = static_cast<bf16*>(v_out);
  return launch_append(a, int64_t(B) * rows, kv->head_dim, dtype, as_stream(stream));
}

LASER_API laser_status laser_kv_check(laser_kv* kv, void* stream) {
  LASER_REQUIRE(kv, "null argument");
  int32_t st = 0;
  LASER_CUDA(cudaMemcpyAsync(&st, kv->status, 4, cudaMemcpyDeviceToHost, as_stream(stream)));
  LASER_CUDA(cudaStreamSynchronize(as_stream(stream)));
  if (st == 0) return LASER_OK;
  LASER_CUDA(cudaMemsetAsync(kv->status, 0, 4, as_stream(stream)));
  set_error(st == LASER_ERR_CAPACITY ? "a sequence outgrew its KV pages" : "a call was given a bad sequence id or parent");
  return st;
}
