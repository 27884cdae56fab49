// Penalties for repeated tokens, biases and grammar masks on the target's rows of a draft tree.
//
// Row 0 of a sequence is the distribution after the committed context, row i + 1 the one after tree node i, so what counts as
// "already there" differs from row to row: the history, and the draft tokens on the path from the root to node i.  For token v
//     c = times v was generated (history past the prompt, and the path),  seen = v in the prompt or c > 0
//     z <- seen ? (z > 0 ? z / rho : z * rho) : z;   z <- z - phi c - pi [c > 0];   z <- z + bias(v);   masked: -inf.
//
// A CTA takes 2048 tokens of the vocabulary and some rows of one sequence.  It counts the history's tokens that fall into its
// range in shared memory (the list is short next to the rows: 16 KB against 8 KB * rows at 4096 tokens), keeps the counts and
// biases of its eight tokens per thread in registers and then streams the rows: one read and one write of each logit, nothing
// else of that size, no workspace.  Draft tokens on a row's path are rare in a CTA's range (a bit set says which nodes matter),
// so they cost a test per row.  Token tid + 256 k belongs to a thread: every access is coalesced whatever the vocabulary's
// alignment, and a warp's 32 tokens share one word of the grammar's mask.  Counts are integers and a token's biases are added
// up by one thread in list order, so a call gives the same bits every time.
#include "logits.cuh"

namespace eagle {

namespace {

constexpr int kLogThreads = 256;
constexpr int kPerThread = 8;
constexpr int kRange = kLogThreads * kPerThread;
constexpr uint32_t kInPrompt = 0x80000000u;

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* base, size_t i) {
  if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(base)[i]) << 16);
  else return static_cast<const float*>(base)[i];
}

template <bool BF16>
__global__ void __launch_bounds__(kLogThreads) logits_kernel(LogitsParams p) {
  __shared__ uint32_t s_count[kRange];
  __shared__ float s_bias[kRange];
  __shared__ int s_btok[kMaxBias];
  __shared__ unsigned long long s_path[kMaxTree];   // nodes on the path of node i whose token lies in this CTA's range
  __shared__ int s_parent[kMaxTree], s_off[kMaxTree];   // parent; place of the node's token in the range, -1: outside
  const int tid = threadIdx.x, b = blockIdx.y, v0 = blockIdx.x * kRange, r_lo = blockIdx.z * p.rows_per_block;
  const bool first = blockIdx.x == 0 && blockIdx.z == 0 && tid == 0;      // reports for the sequence

  // ---- the tree
  const int n = p.tree_sizes ? p.tree_sizes[p.shared_tree ? 0 : b] : p.T;
  bool bad = n < 0 || n > p.T;
  {
    int wrong = 0, off = -1;
    if (!bad && tid < n) {
      const int m = p.tree_parent[(p.shared_tree ? 0 : static_cast<size_t>(b) * p.T) + tid], t = p.draft_tokens[static_cast<size_t>(b) * p.T + tid];
      wrong = m < -1 || m >= tid;
      if (t < 0 || t >= p.V) { if (blockIdx.x == 0 && blockIdx.z == 0) report_status(p.status, EAGLE_ERR_TOKEN); }
      else if (t >= v0 && t < v0 + kRange) off = t - v0;
      s_parent[tid] = m;
      s_off[tid] = off;
    }
    bad = __syncthreads_or(bad || wrong);
  }
  const int rows = bad ? p.T + 1 : n + 1, r_hi = min(rows, r_lo + p.rows_per_block);
  const size_t row0 = static_cast<size_t>(b) * (p.T + 1) * p.V;
  if (bad) {
    if (first) report_status(p.status, EAGLE_ERR_TREE);
    for (int r = r_lo; r < r_hi; ++r)
      for (int k = 0; k < kPerThread; ++k) {
        const int v = v0 + tid + k * kLogThreads;
        if (v < p.V) p.out[row0 + static_cast<size_t>(r) * p.V + v] = 0.f;
      }
    return;
  }
  if (r_lo >= r_hi) return;

  // ---- history: counts of the tokens in the range
  for (int i = tid; i < kRange; i += kLogThreads) { s_count[i] = 0u; s_bias[i] = 0.f; }
  if (tid < n) {
    unsigned long long path = 0ull;
    for (int m = tid; m >= 0; m = s_parent[m])
      if (s_off[m] >= 0) path |= 1ull << m;
    s_path[tid] = path;
  }
  const int nb = p.bias_tokens ? min(max(p.bias_len ? p.bias_len[b] : p.max_bias, 0), p.max_bias) : 0;
  for (int i = tid; i < nb; i += kLogThreads) s_btok[i] = p.bias_tokens[static_cast<size_t>(b) * p.max_bias + i];
  __syncthreads();
  if (p.history) {
    const int len = min(max(p.history_len[b], 0), p.H), prompt = p.prompt_len ? p.prompt_len[b] : 0;
    const int32_t* h = p.history + static_cast<size_t>(b) * p.H;
    for (int i = tid; i < len; i += kLogThreads) {
      const int t = h[i];
      if (t < 0 || t >= p.V) { if (blockIdx.x == 0 && blockIdx.z == 0) report_status(p.status, EAGLE_ERR_TOKEN); }
      else if (t >= v0 && t < v0 + kRange) {
        if (i < prompt) atomicOr(&s_count[t - v0], kInPrompt);
        else atomicAdd(&s_count[t - v0], 1u);
      }
    }
  }
  for (int i = tid; i < nb; i += kLogThreads) {
    const int t = s_btok[i];
    if (t < 0 || t >= p.V) { if (blockIdx.x == 0 && blockIdx.z == 0) report_status(p.status, EAGLE_ERR_TOKEN); continue; }
    if (t < v0 || t >= v0 + kRange) continue;
    bool mine = true;                                // the first entry of a token adds up all of them
    for (int j = 0; j < i; ++j) mine = mine && s_btok[j] != t;
    if (!mine) continue;
    float sum = 0.f;
    for (int j = i; j < nb; ++j)
      if (s_btok[j] == t) sum += p.bias_values[static_cast<size_t>(b) * p.max_bias + j];
    s_bias[t - v0] = sum;
  }
  __syncthreads();

  uint32_t count[kPerThread];
  float bias[kPerThread];
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    count[k] = s_count[tid + k * kLogThreads];
    bias[k] = s_bias[tid + k * kLogThreads];
  }
  const float rho = p.repetition ? p.repetition[b] : 1.f, pi = p.presence ? p.presence[b] : 0.f, phi = p.frequency ? p.frequency[b] : 0.f;
  const int words = (p.V + 31) / 32;

  // ---- rows, the next one's logits on their way while one is worked on
  float z[kPerThread], next[kPerThread];
  auto fetch = [&](int r, float* to) {
    const size_t at = row0 + static_cast<size_t>(r) * p.V + v0 + tid;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k)
      if (v0 + tid + k * kLogThreads < p.V) to[k] = load_logit<BF16>(p.logits, at + k * kLogThreads);
  };
  fetch(r_lo, z);
  for (int r = r_lo; r < r_hi; ++r) {
    if (r + 1 < r_hi) fetch(r + 1, next);
    uint32_t extra[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) extra[k] = 0u;
    for (unsigned long long path = r > 0 ? s_path[r - 1] : 0ull; path; path &= path - 1) {
      const int off = s_off[__ffsll(static_cast<long long>(path)) - 1];
      if ((off & (kLogThreads - 1)) == tid) {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) extra[k] += (off >> 8) == k;
      }
    }
    const size_t at = row0 + static_cast<size_t>(r) * p.V + v0 + tid;
    const uint32_t* mask = p.allowed ? p.allowed + (static_cast<size_t>(b) * (p.T + 1) + r) * words : nullptr;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int v = v0 + tid + k * kLogThreads;
      if (v >= p.V) continue;
      float x = z[k];
      const uint32_t c = (count[k] & ~kInPrompt) + extra[k];
      if (c | (count[k] & kInPrompt)) {
        x = x > 0.f ? __fdiv_rn(x, rho) : x * rho;
        if (c) x = x - phi * static_cast<float>(c) - pi;
      }
      x += bias[k];
      if (mask && !((__ldg(mask + (v >> 5)) >> (v & 31)) & 1u)) x = -INFINITY;
      p.out[at + k * kLogThreads] = x;
    }
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) z[k] = next[k];
  }
}

}  // namespace

cudaError_t launch_logits(const LogitsParams& p_in, int sm_count, cudaStream_t stream) {
  LogitsParams p = p_in;
  const int ranges = (p.V + kRange - 1) / kRange, rows = p.T + 1;
  // rows are shared out over several CTAs (which count the history again each) while there are too few to fill the machine
  int splits = 1;
  while (static_cast<long long>(ranges) * p.B * splits < 8ll * sm_count && splits < rows) ++splits;
  p.rows_per_block = (rows + splits - 1) / splits;
  const dim3 grid(static_cast<unsigned>(ranges), static_cast<unsigned>(p.B), static_cast<unsigned>((rows + p.rows_per_block - 1) / p.rows_per_block));
  if (p.bf16) logits_kernel<true><<<grid, kLogThreads, 0, stream>>>(p);
  else logits_kernel<false><<<grid, kLogThreads, 0, stream>>>(p);
  count_launch();
  return cudaGetLastError();
}

}  // namespace eagle
