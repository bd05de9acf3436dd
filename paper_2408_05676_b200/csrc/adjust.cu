// What is done to the logits of a verify step before acceptance: penalties for tokens that the text has already, biases, and the tokens
// that a grammar allows.  For row i and token v, with n how often v occurs in the generated part of the text and among the drafts on the
// row's path (rows 1 .. i of a chain, the ancestors and itself in a token tree):
//   x = logit;  v in the text or on the path: x = x > 0 ? x / repetition : x * repetition
//   x = x - frequency n - presence [n > 0];  x = x + bias(v);  v not allowed: x = -inf
//
// A CTA takes a run of the vocabulary for all rows of one sequence.  It counts the text's tokens of its run in shared memory (whole
// numbers, whose order does not matter), notes which rows' tokens a token is as a 64-bit mask, and adds up its biases in the order of the
// list; then the rows pass by: one load and one store a logit, coalesced whatever the rows' alignment, and the tables only where a token
// has an entry.  A warp's 32 tokens are one word of the grammar mask, and logits that it forbids are not read.
// Bound by memory where rows are many; with few rows by the counting (each CTA reads the text) and the launch.
#include "model.cuh"
#include "tree.cuh"

namespace laser {
namespace {

constexpr int kThreads = 256;

struct AdjustArgs {
  const float* logits;
  float* out;
  const int32_t *tokens, *parents, *n_rows, *hist, *hist_len, *prompt_len;
  long long hist_stride;
  const float *repetition, *frequency, *presence;
  const int32_t *bias_offsets, *bias_ids;
  const float* bias_values;
  const uint32_t* allowed;
  long long mask_seq_stride, mask_row_stride;
  int R, V;
};

// U: tokens of a thread
template <int U>
__global__ void __launch_bounds__(kThreads)
adjust_kernel(const AdjustArgs a) {
  constexpr int C = U * kThreads;
  __shared__ uint32_t s_count[C];              // occurrences in the generated text; top bit: one in the prompt
  __shared__ unsigned long long s_rows[C];     // rows of the step whose token it is
  __shared__ float s_bias[C];
  __shared__ unsigned long long s_path[64];
  __shared__ int s_id[kThreads];
  __shared__ float s_val[kThreads];
  next_may_launch();
  const int b = blockIdx.y, v0 = blockIdx.x * C, tid = threadIdx.x, lane = tid & 31;
#pragma unroll
  for (int k = 0; k < U; ++k) { s_count[k * kThreads + tid] = 0; s_rows[k * kThreads + tid] = 0; s_bias[k * kThreads + tid] = 0.f; }
  wait_for_earlier();
  const int nr = min(max(a.n_rows[b], 0), a.R);
  if (nr == 0) return;
  __syncthreads();
  if (tid < 32) {
    unsigned long long mask[2];
    if (a.parents) {
      tree_paths(a.parents + size_t(b) * a.R, nr, lane, mask);
    } else {
      mask[0] = (2ull << lane) - 1;
      mask[1] = (2ull << (lane + 32)) - 1;     // (row 63: all ones)
    }
    s_path[lane] = mask[0] & ~1ull;            // the pending token, row 0, is in the text
    s_path[lane + 32] = mask[1] & ~1ull;
  }
  const int len = a.hist ? int(min((long long)max(a.hist_len[b], 0), a.hist_stride)) : 0, made = a.prompt_len ? a.prompt_len[b] : 0;
  const int32_t* text = a.hist + size_t(b) * a.hist_stride;
#pragma unroll 4
  for (int j = tid; j < len; j += kThreads) {
    const unsigned at = unsigned(text[j]) - unsigned(v0);
    if (at < unsigned(C)) {
      if (j >= made) atomicAdd(&s_count[at], 1u);
      else atomicOr(&s_count[at], 0x80000000u);
    }
  }
  if (tid > 0 && tid < nr) {
    const unsigned at = unsigned(a.tokens[size_t(b) * a.R + tid]) - unsigned(v0);
    if (at < unsigned(C)) atomicOr(&s_rows[at], 1ull << tid);
  }
  if (a.bias_offsets) {
    const int from = a.bias_offsets[b], to = a.bias_offsets[b + 1];
    for (int j0 = from; j0 < to; j0 += kThreads) {
      __syncthreads();
      s_id[tid] = j0 + tid < to ? a.bias_ids[j0 + tid] : -1;
      s_val[tid] = j0 + tid < to ? a.bias_values[j0 + tid] : 0.f;
      __syncthreads();
      if (tid < 32) {
        for (int x = 0; x < min(kThreads, to - j0); x += 32) {
          const int id = s_id[x + lane];
          const unsigned at = unsigned(id) - unsigned(v0);
          const bool here = id >= 0 && at < unsigned(C);
          if (!__any_sync(0xffffffffu, here)) continue;
          // entries of one token are added in the list's order
          const unsigned same = __match_any_sync(0xffffffffu, here ? int(at) : -1);
          const int turn = __popc(same & ((1u << lane) - 1)), turns = __reduce_max_sync(0xffffffffu, here ? turn : 0);
          for (int y = 0; y <= turns; ++y) {
            if (here && turn == y) s_bias[at] += s_val[x + lane];
            __syncwarp();
          }
        }
      }
    }
  }
  __syncthreads();
  uint32_t some = 0, inside = 0;      // of the thread's tokens: those that something is done to; those of the vocabulary
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int at = k * kThreads + tid;
    if (s_count[at] != 0 || s_rows[at] != 0 || s_bias[at] != 0.f) some |= 1u << k;      // (a NaN is some bias)
    if (v0 + at < a.V) inside |= 1u << k;
  }
  const float rep = a.repetition ? a.repetition[b] : 1.f, freq = a.frequency ? a.frequency[b] : 0.f, pres = a.presence ? a.presence[b] : 0.f;
  // a row's logits are requested while the one before is finished, its words of the mask one row earlier still (lane k: the warp's k-th word)
  const float* in = a.logits + size_t(b) * a.R * a.V + v0 + tid;
  float* out = a.out + size_t(b) * a.R * a.V + v0 + tid;
  const int word = (v0 >> 5) + lane * (kThreads / 32) + (tid >> 5);
  const bool has_word = a.allowed && lane < U && (word << 5) < a.V;
  const uint32_t* words = a.allowed + b * a.mask_seq_stride + word;
  auto mask = [&](int i) { return has_word && i < nr ? words[i * a.mask_row_stride] : 0u; };
  auto fetch = [&](const float* from, uint32_t w, uint32_t& on, float (&x)[U]) {
    on = inside;
    if (a.allowed) {
      uint32_t bits = 0;
#pragma unroll
      for (int k = 0; k < U; ++k) bits |= (__shfl_sync(0xffffffffu, w, k) >> lane & 1u) << k;      // (a token is lane mod 32)
      on &= bits;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) x[k] = on >> k & 1u ? from[k * kThreads] : -INFINITY;
  };
  uint32_t next_word = mask(0), on, next_on = 0;
  float x[U], next[U];
  fetch(in, next_word, on, x);
  next_word = mask(1);
  for (int i = 0; i < nr; ++i) {
    in += a.V;
    if (i + 1 < nr) {
      fetch(in, next_word, next_on, next);
      next_word = mask(i + 2);
    }
    if (some & on) {
      const unsigned long long path = s_path[i];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (!((some & on) >> k & 1u)) continue;
        const uint32_t count = s_count[k * kThreads + tid];
        const int drafts = __popcll(s_rows[k * kThreads + tid] & path), n = int(count & 0x7fffffffu) + drafts;
        if (count != 0 || drafts != 0) x[k] = x[k] > 0.f ? __fdiv_rn(x[k], rep) : __fmul_rn(x[k], rep);
        if (n > 0) x[k] = __fsub_rn(__fsub_rn(x[k], __fmul_rn(freq, float(n))), pres);
        x[k] = __fadd_rn(x[k], s_bias[k * kThreads + tid]);
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (inside >> k & 1u) out[k * kThreads] = x[k];
    out += a.V;
#pragma unroll
    for (int k = 0; k < U; ++k) x[k] = next[k];
    on = next_on;
  }
}

}  // namespace
}  // namespace laser

using namespace laser;

LASER_API laser_status laser_adjust_logits(const float* logits, const int32_t* tokens, const int32_t* parents, const int32_t* n_rows,
                                           const int32_t* hist, const int32_t* hist_len, int64_t hist_stride, const int32_t* prompt_len,
                                           const float* repetition, const float* frequency, const float* presence, const int32_t* bias_offsets,
                                           const int32_t* bias_ids, const float* bias_values, const uint32_t* allowed, int64_t mask_seq_stride,
                                           int64_t mask_row_stride, int32_t B, int32_t rows, int32_t V, float* out, void* stream) {
  LASER_REQUIRE(logits && out && tokens && n_rows, "null argument");
  LASER_REQUIRE(B >= 0 && B <= 65535, "B = %d outside [0, 65535]", B);
  LASER_REQUIRE(rows >= 1 && rows <= 64, "rows = %d outside [1, 64]", rows);
  LASER_REQUIRE(V >= 1 && V <= (1 << 30), "V = %d", V);
  LASER_REQUIRE(!hist || (hist_len && hist_stride >= 0 && hist_stride <= INT32_MAX), "hist needs hist_len and a stride");
  LASER_REQUIRE((!bias_offsets && !bias_ids && !bias_values) || (bias_offsets && bias_ids && bias_values), "the three bias arrays go together");
  const int64_t n_words = (int64_t(V) + 31) / 32;
  LASER_REQUIRE(!allowed || ((mask_row_stride == 0 || mask_row_stride >= n_words) && (mask_seq_stride == 0 || mask_seq_stride >= n_words)),
                "mask strides of less than the %lld words of a row", (long long)n_words);
  LASER_REQUIRE(((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(allowed)) & 3) == 0, "arrays must be 4-byte aligned");
  const size_t bytes = size_t(B) * rows * V * 4;
  const uintptr_t from = reinterpret_cast<uintptr_t>(logits), to = reinterpret_cast<uintptr_t>(out);
  LASER_REQUIRE(from == to || from + bytes <= to || to + bytes <= from, "out overlaps logits without being the same array");
  if (B == 0) return LASER_OK;
  AdjustArgs a{logits, out, tokens, parents, n_rows, hist, hist_len, prompt_len, hist_stride, repetition, frequency, presence,
               bias_offsets, bias_ids, bias_values, allowed, mask_seq_stride, mask_row_stride, rows, V};
  // runs of 2048 tokens; of 512 where the SMs would be left without work
  if (int64_t(B) * ceil_div(V, 8 * kThreads) >= 148)
    LASER_CUDA(launch_overlapped(adjust_kernel<8>, dim3(unsigned(ceil_div(V, 8 * kThreads)), unsigned(B)), kThreads, 0, as_stream(stream), a));
  else
    LASER_CUDA(launch_overlapped(adjust_kernel<2>, dim3(unsigned(ceil_div(V, 2 * kThreads)), unsigned(B)), kThreads, 0, as_stream(stream), a));
  count_launch();
  return LASER_OK;
}
