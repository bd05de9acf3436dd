// What is done to the logits of a verify step before acceptance: penalties for tokens that the text has already, biases, and the tokens
// that a grammar allows.  For row i and token v, with n how often v occurs in the generated part of the text and among the drafts on the
// row's path (rows 1 .. i of a chain, the ancestors and itself in a token tree):
//   x = logit;  v in the text or on the path: x = x > 0 ? x / repetition : x * repetition
//   x = x - frequency n - presence [n > 0];  x = x + bias(v);  v not allowed: x = -inf
//
// A CTA takes a run of the vocabulary for all rows of one sequence.  It counts the text's tokens of its run in shared memory (whole
// numbers, whose order does not matter), notes which rows' tokens a token is as a 64-bit mask, and adds up its biases in the order of the
// list; what that means for a row's logits is a factor and a difference a token, but for the step's own drafts.  Then the rows pass by, a
// load and a store a logit, or four of them where all rows begin on 16 bytes (64 x 9 rows of 32000: 19.2 us instead of 25.2).  A trip to
// memory takes 1.6 us under load, so each thread has its logits of the next kAhead rows on their way into shared memory (72 KB an SM; with
// one row ahead, in registers, 64 trees of 17 rows took 71 us instead of 66).  32 tokens are one word of the grammar mask, and logits
// that it forbids are not read (of four, if it forbids them all).
// Times (us; floors by bytes at 6.56 TB/s in brackets): one row of 32000 2.3 (0.04), 64 x 9 rows of 32000 19.2 (12.7), 64 trees of 17 rows
// of 50257 62 (36): bound by the instructions of 4-byte accesses, 42 % of the LSU's and 54 % of the logic pipe's cycles.
#include <type_traits>

#include "model.cuh"
#include "tma.cuh"
#include "tree.cuh"

namespace laser {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 3;

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

__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// U: tokens of a thread
template <int U>
struct Tables {
  static constexpr int C = U * kThreads;
  unsigned long long rows[C];     // rows of the step whose token it is
  uint32_t count[C];              // occurrences in the generated text; top bit: one in the prompt
  float bias[C];
  float x[kAhead][C];             // logits of the next rows
  uint32_t words[2 * kAhead][C / 32];   // and their words of the mask, twice as far ahead
  unsigned long long path[64];
  int id[kThreads];
  float val[kThreads];
};

// N: tokens of a thread that lie side by side, fetched and stored together: 4 where all rows begin on 16 bytes, else 1
template <int U, int N>
__global__ void __launch_bounds__(kThreads, 3)
adjust_kernel(const AdjustArgs a) {
  using S = Tables<U>;
  static_assert(N == 1 || (N == 4 && U % 4 == 0), "vectors of four");
  constexpr int C = S::C, kFirst = 4;
  extern __shared__ __align__(16) uint8_t smem[];
  S& s = *reinterpret_cast<S*>(smem);
  next_may_launch();
  const int b = blockIdx.y, v0 = blockIdx.x * C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto place = [&](int k) { return k / N * (N * kThreads) + tid * N + k % N; };      // of the thread's token k in the run
#pragma unroll
  for (int k = 0; k < U; ++k) { s.count[k * kThreads + tid] = 0; s.rows[k * kThreads + tid] = 0; s.bias[k * kThreads + tid] = 0.f; }
  wait_for_earlier();
  // ---- what is read before the rows, in two trips to memory: the sequence's numbers and the first rows' words of the mask; then the first of
  // its text, biases and drafts, and the first rows ----
  const int word = lane / N * (N * kThreads / 32) + warp * N + lane % N;                   // a lane's word: one of the U of the warp's tokens
  const bool has_word = a.allowed && lane < U && v0 + (word << 5) < a.V;
  const uint32_t* const words = a.allowed + b * a.mask_seq_stride + (v0 >> 5) + word;
  auto get_words = [&](int i) { if (has_word && i < a.R) copy4(smem_u32(&s.words[i % (2 * kAhead)][word]), words + i * a.mask_row_stride); };
#pragma unroll
  for (int i = 0; i < 2 * kAhead; ++i) get_words(i);
  copies_commit();
  const int n_rows = a.n_rows[b];
  const int hist_len = a.hist ? a.hist_len[b] : 0, made = a.prompt_len ? a.prompt_len[b] : 0;
  const int bias_from = a.bias_offsets ? a.bias_offsets[b] : 0, bias_to = a.bias_offsets ? a.bias_offsets[b + 1] : 0;
  const float rep = a.repetition ? a.repetition[b] : 1.f, freq = a.frequency ? a.frequency[b] : 0.f, pres = a.presence ? a.presence[b] : 0.f;
  const int nr = min(max(n_rows, 0), a.R), len = int(min((long long)max(hist_len, 0), a.hist_stride));
  copies_wait<0>();
  if (nr == 0) return;
  __syncwarp();
  uint32_t inside = 0;                         // the thread's tokens that are of the vocabulary
#pragma unroll
  for (int k = 0; k < U; ++k) if (v0 + place(k) < a.V) inside |= 1u << k;
  auto allowed = [&](int i) {                  // those that row i may have
    if (!a.allowed) return inside;
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < U; k += N)
      bits |= (s.words[i % (2 * kAhead)][k / N * (N * kThreads / 32) + warp * N + lane * N / 32] >> (lane * N % 32) & ((1u << N) - 1)) << k;
    return bits & inside;
  };
  const float* in = a.logits + size_t(b) * a.R * a.V + v0 + tid * N;      // of the next row to be requested
  uint32_t on[kAhead];                         // what the next rows may have
  auto get_row = [&](int i) {
    uint32_t bits = 0;
    if (i < nr) {
      bits = allowed(i);
      const uint32_t at = smem_u32(&s.x[i % kAhead][tid * N]);
#pragma unroll
      for (int k = 0; k < U; k += N) {
        if (!(bits >> k & ((1u << N) - 1))) continue;
        if (N == 4) copy16(at + k * (kThreads * 4), in + k * kThreads);
        else copy4(at + k * (kThreads * 4), in + k * kThreads);
      }
    }
    in += a.V;
    return bits;
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    on[i] = get_row(i);
    copies_commit();
  }
  const int32_t* const text = a.hist + size_t(b) * a.hist_stride;
  int tok[kFirst];
#pragma unroll
  for (int u = 0; u < kFirst; ++u) tok[u] = tid + u * kThreads < len ? text[tid + u * kThreads] : -1;
  const int draft = tid > 0 && tid < nr ? a.tokens[size_t(b) * a.R + tid] : -1;
  int id = bias_from + tid < bias_to ? a.bias_ids[bias_from + tid] : -1;
  float val = bias_from + tid < bias_to ? a.bias_values[bias_from + tid] : 0.f;
  if (warp == 0) {
    unsigned long long path[2];
    if (a.parents) {
      tree_paths(a.parents + size_t(b) * a.R, nr, lane, path);
    } else {
      path[0] = (2ull << lane) - 1;
      path[1] = (2ull << (lane + 32)) - 1;     // (row 63: all ones)
    }
    s.path[lane] = path[0] & ~1ull;            // the pending token, row 0, is in the text
    s.path[lane + 32] = path[1] & ~1ull;
  }

  // ---- the tables ----
  __syncthreads();
  auto count = [&](int token, int j) {
    const unsigned at = unsigned(token) - unsigned(v0);
    if (at < unsigned(C)) {
      if (j >= made) atomicAdd(&s.count[at], 1u);
      else atomicOr(&s.count[at], 0x80000000u);
    }
  };
#pragma unroll
  for (int u = 0; u < kFirst; ++u) count(tok[u], tid + u * kThreads);
#pragma unroll 4
  for (int j = tid + kFirst * kThreads; j < len; j += kThreads) count(text[j], j);
  {
    const unsigned at = unsigned(draft) - unsigned(v0);
    if (at < unsigned(C)) atomicOr(&s.rows[at], 1ull << tid);
  }
  for (int j0 = bias_from; j0 < bias_to; j0 += kThreads) {
    if (j0 > bias_from) {
      __syncthreads();
      id = j0 + tid < bias_to ? a.bias_ids[j0 + tid] : -1;
      val = j0 + tid < bias_to ? a.bias_values[j0 + tid] : 0.f;
    }
    s.id[tid] = id;
    s.val[tid] = val;
    __syncthreads();
    if (warp == 0) {
#pragma unroll 1
      for (int x0 = 0; x0 < min(kThreads, bias_to - j0); x0 += 32) {
        const unsigned at = unsigned(s.id[x0 + lane]) - unsigned(v0);
        const bool here = at < unsigned(C);
        if (!__any_sync(0xffffffffu, here)) continue;
        // entries of one token are added in the list's order
        const unsigned same = __match_any_sync(0xffffffffu, here ? int(at) : -1);
        const int turn = __popc(same & ((1u << lane) - 1)), turns = __reduce_max_sync(0xffffffffu, here ? turn : 0);
        for (int y = 0; y <= turns; ++y) {
          if (here && turn == y) s.bias[at] += s.val[x0 + lane];
          __syncwarp();
        }
      }
    }
  }
  __syncthreads();
  // of the thread's tokens: those of the text, what is taken from them (all three terms as one), and those that are drafts, few
  // enough for a branch
  uint32_t seen = 0, drafted = 0;
  float less[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int at = place(k);
    const uint32_t c = s.count[at];
    const float n = float(c & 0x7fffffffu);
    less[k] = (freq * n + (n > 0.f ? pres : 0.f)) - s.bias[at];
    if (s.rows[at] != 0) { drafted |= 1u << k; less[k] = 0.f; }
    else if (c != 0) seen |= 1u << k;
  }
  const float inv = 1.f / rep;

  // ---- the rows ----
  float* out = a.out + size_t(b) * a.R * a.V + v0 + tid * N;
#pragma unroll 1
  for (int i = 0; i < nr; ++i) {
    copies_wait<kAhead - 1>();
    __syncwarp();
    float x[U];
#pragma unroll
    for (int k = 0; k < U; k += N) {
      const float* from = &s.x[i % kAhead][place(k)];
      if (N == 4) *reinterpret_cast<float4*>(&x[k]) = *reinterpret_cast<const float4*>(from);
      else x[k] = *from;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float f = x[k] > 0.f ? inv : rep, y = x[k] * (seen >> k & 1u ? f : 1.f) - less[k];
      x[k] = on[0] >> k & 1u ? y : -INFINITY;
    }
    if (drafted & on[0]) {
      const unsigned long long path = s.path[i];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (!((drafted & on[0]) >> k & 1u)) continue;
        const uint32_t c = s.count[place(k)];
        const int drafts = __popcll(s.rows[place(k)] & path);
        const float n = float(int(c & 0x7fffffffu) + drafts);
        if (c != 0 || drafts != 0) x[k] *= x[k] > 0.f ? inv : rep;
        x[k] -= (freq * n + (n > 0.f ? pres : 0.f)) - s.bias[place(k)];
      }
    }
#pragma unroll
    for (int k = 0; k < U; k += N) {
      if (!(inside >> k & 1u)) continue;
      if (N == 4) *reinterpret_cast<float4*>(out + k * kThreads) = *reinterpret_cast<const float4*>(&x[k]);
      else out[k * kThreads] = x[k];
    }
    out += a.V;
#pragma unroll
    for (int y = 0; y + 1 < kAhead; ++y) on[y] = on[y + 1];
    get_words(i + 2 * kAhead);          // (in the place of this row's, which were read before the last __syncwarp)
    on[kAhead - 1] = get_row(i + kAhead);
    copies_commit();
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
  auto launch = [&](auto tokens_of_thread, auto together) -> laser_status {
    constexpr int U = decltype(tokens_of_thread)::value, N = decltype(together)::value;
    LASER_CUDA((allow_shared_memory<adjust_kernel<U, N>>(int(sizeof(Tables<U>)))));
    LASER_CUDA(launch_overlapped(adjust_kernel<U, N>, dim3(unsigned(ceil_div(V, U * kThreads)), unsigned(B)), kThreads, sizeof(Tables<U>), as_stream(stream), a));
    return LASER_OK;
  };
  // runs of 2048 tokens; of 512 where the SMs would be left without work
  const bool fours = V % 4 == 0 && ((from | to) & 15) == 0;
  const std::integral_constant<int, 1> one;
  if (int64_t(B) * ceil_div(V, 8 * kThreads) < 148) LASER_TRY(launch(std::integral_constant<int, 2>{}, one));
  else if (fours) LASER_TRY(launch(std::integral_constant<int, 8>{}, std::integral_constant<int, 4>{}));
  else LASER_TRY(launch(std::integral_constant<int, 8>{}, one));
  count_launch();
  return LASER_OK;
}
