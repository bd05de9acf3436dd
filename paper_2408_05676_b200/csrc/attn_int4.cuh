// What the attention kernels over the 4-bit cache share: their arguments and small device functions.
#pragma once
#include "int4.cuh"
#include "mma.cuh"
#include "model.cuh"
#include "tma.cuh"
#include "tree.cuh"

namespace laser {

constexpr int kAttnInt4Seqs = 1024;    // sequences (or prompt chunks) of a call: their offsets are in shared memory
constexpr float kNothing = 1e30f;      // -m of rows that have seen nothing

struct AttnArgs {
  // rows: from a step's tables (row_ctx, row_n) or the sequences' lengths; parents: a token tree's (up to 64 rows)
  const int32_t *seq_ids, *row_ctx, *row_n, *n_rows, *seq_len, *parents;
  int B, Rs, max_seqs, capacity, Hkv, G;       // G: query heads of a kv head
  const int32_t* page_table;
  int pages_per_seq;
  const uint8_t* pages;                        // this layer's
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  long long ldq, ldo;                          // elements between rows
  int vec_out;                                 // rows of out are 16-byte aligned
  unsigned group_inv;                          // 2^32 / G rounded up (G > 1)
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
// two codes at bits 3 .. 6 of the halves -> the two values.  (w & 0x00780078) | 0x41804180 as one instruction: of two constants the
// compiler makes two, and the kernel's busiest pipe is the one for logic and shifts.
__device__ __forceinline__ uint32_t values(uint32_t w, uint32_t s2, uint32_t z2) {
  uint32_t u;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(w), "r"(0x00780078u), "r"(0x41804180u));
  return fma2(u, s2, z2);
}
__device__ __forceinline__ void copy_block(uint32_t dst, const void* src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// head_dim 128: tensor-memory kernel.  Partial results of `ctas` CTAs take part_floats.
laser_status attn_int4_wide_launch(const AttnArgs& a, int ctas, cudaStream_t stream);
size_t attn_int4_wide_part_floats(int ctas);

}  // namespace laser
